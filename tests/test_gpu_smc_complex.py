"""Consolidation of complex states: (re, im) pairs, in complex64 or fp32 tensors on either side, give the same bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("table_complex", [False, True])
@pytest.mark.parametrize("states_complex", [False, True])
def test_pairs_are_pairs(cuda_device, table_complex, states_complex):
    import torch
    import paper_2608_02560_gb300 as pg
    gen = torch.Generator(device=cuda_device).manual_seed(4)
    semantic = torch.randn((5, 2, 8, 16), dtype=torch.complex64, device=cuda_device, generator=gen)
    states = torch.randn((7, 2, 8, 16), dtype=torch.complex64, device=cuda_device, generator=gen)
    slots = torch.tensor([4, 0, -1, 4, 2, 0, 4], device=cuda_device)
    want = semantic.clone()
    for c, s in enumerate(slots.tolist()):
        if s >= 0:
            want[s] = 0.7 * want[s] + 0.3 * states[c]
    real = torch.view_as_real
    pg.precog_smc_consolidate(semantic if table_complex else real(semantic), states if states_complex else real(states), slots, 0.3)
    assert pg.precog_device_status()[0] == 0
    # three deposits at most: three roundings each of the two products and their sum
    assert float((real(semantic) - real(want)).abs().max()) <= 9 * 2.0 ** -24 * 8
    with pytest.raises(ValueError, match="resolve_conj"):
        pg.precog_smc_consolidate(real(semantic), states.conj(), slots, 0.3)
    with pytest.raises(ValueError, match="resolve_conj"):
        pg.precog_smc_consolidate(semantic.conj(), states, slots, 0.3)
