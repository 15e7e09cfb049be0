"""Banks and windows with nothing in them. torch gives an empty tensor the address 0, which the convolution's C call
reads as "nothing came before": sequences that have no entry or layer to go by are refused, not started from zeros."""
import pytest


@pytest.fixture
def pg(monkeypatch):
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    monkeypatch.setattr(pg, "_stream_on", lambda device, stream: None)
    return pg


def _rows(n):
    import torch
    return dict(x=torch.zeros(n, 8), weight=torch.zeros(8, 4), offsets=torch.tensor([0, 2, n] if n else [0]), y_out=torch.zeros(n, 8))


@pytest.mark.parametrize("entries", [0, 1])
def test_fewer_entries_than_sequences(pg, entries):
    import torch
    with pytest.raises((ValueError, pg.PrecogError), match="bank has fewer rows than sequences"):
        pg.precog_causal_conv(**_rows(6), bank=torch.zeros(entries, 1, 3, 8))
    pg.precog_causal_conv(**_rows(0), bank=torch.zeros(entries, 1, 3, 8))


@pytest.mark.parametrize("bank_layers,out_layers", [(0, None), (None, 0), (0, 0)])
def test_a_table_without_layers_has_no_layer_0(pg, bank_layers, out_layers):
    import torch
    table = lambda layers: None if layers is None else torch.zeros(2, layers, 3, 8)  # noqa: E731
    for idx in (None,) if bank_layers is None else (None, torch.tensor([0, 1])):
        with pytest.raises(pg.PrecogError, match="layer"):
            pg.precog_causal_conv(**_rows(6), bank=table(bank_layers), windows_out=table(out_layers), idx=idx)
