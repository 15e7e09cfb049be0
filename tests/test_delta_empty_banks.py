"""A bank of matrix states with nothing in it has no address, which the C call reads as "from zero states": sequences
that have no entry or layer to go by are refused."""
import pytest


@pytest.mark.parametrize("entries,layers", [(0, 1), (1, 1), (2, 0), (0, 0)])
def test_delta_scan(entries, layers):
    import torch
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    inputs = pg.DeltaInputs(1, 1, 8, 8, pg.PRECOG_F32, 1.0, 16, 16, 16, 16, 16, 8, 8, 8)
    inputs.rows = 6
    with pytest.raises(ValueError, match="bank has no"):
        pg.precog_delta_scan(inputs, torch.tensor([0, 2, 6]), 6, bank=torch.zeros(entries, layers, 1, 8, 8), y_out=torch.zeros(6, 1, 8))
