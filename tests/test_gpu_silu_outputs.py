"""SiLU where bf16 rows go into fp32 outputs: those are not rounded to 16 bits, so the gate is as exact as for fp32
rows. An exponential within 2 units of 2^-23, a sum and a quotient of half a unit each: 3 units, under 8 * 2^-24 of
the value. All else in these calls is exact (products with 1, sums with 0)."""
import numpy as np
import pytest

import oracle
from tests._util import to_np

pytestmark = pytest.mark.gpu
BOUND = 8 * 2.0 ** -24


def _gates(dev, T, D):
    import torch
    gen = torch.Generator(device=dev).manual_seed(T + D)
    return (120 * torch.rand((T, D), device=dev, generator=gen) - 60).bfloat16()


def _within(got, gate):
    ref = oracle.silu(to_np(gate))
    assert np.abs(ref).min() > 1e-30 or (np.abs(ref).min() == 0 and (to_np(gate)[ref == 0] == 0).all())
    assert float((np.abs(to_np(got) - ref) - BOUND * np.abs(ref)).max()) <= 0.0


@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("T,D", [(40, 64), (9, 1032), (7, 2048), (5, 4096), (3, 8200)])
def test_a_gate_into_an_fp32_residual(cuda_device, first, T, D):
    import torch
    import paper_2608_02560_gb300 as pg
    gate, x = _gates(cuda_device, T, D), torch.ones((T, D), dtype=torch.bfloat16, device=cuda_device)
    h = torch.zeros((T, D), device=cuda_device)
    pg.precog_block_norm(x, gate=gate, gate_first=first, residual=h, residual_out=h, norm="none")
    assert pg.precog_device_status()[0] == 0
    _within(h, gate)


@pytest.mark.parametrize("cplx", [False, True])
@pytest.mark.parametrize("n,D", [(1, 64), (5, 1032)])
def test_a_gate_into_an_fp32_readout(cuda_device, cplx, n, D):
    import torch
    import paper_2608_02560_gb300 as pg
    d, N = cuda_device, 16
    gate, one = _gates(d, n, D)[None], torch.ones((1, n, D), dtype=torch.bfloat16, device=d)
    nothing = torch.zeros((1, n, N), dtype=torch.bfloat16, device=d)
    kind = torch.complex64 if cplx else torch.float32
    A, h = -torch.ones((1, D, N), dtype=kind, device=d), torch.zeros((n, 1, D, N), dtype=kind, device=d)
    y = torch.empty((1, n, D), device=d)
    inputs = pg.scan_inputs(one, one, nothing, A, nothing, a_kind=pg.PRECOG_A_COMPLEX if cplx else pg.PRECOG_A_GENERAL)
    pg.precog_scan_step(inputs, h, skip=torch.ones((1, D), device=d), gate=gate, y_out=y)
    assert pg.precog_device_status()[0] == 0
    _within(y[0], gate[0])


def test_every_bf16_gate(cuda_device):
    """All 65,536: NaN and -infinity give NaN, infinity stays, and below -87, where 87 e^-87 < 2e-36, 0 is as good."""
    import torch
    import paper_2608_02560_gb300 as pg
    gate = torch.arange(-32768, 32768, device=cuda_device).short().view(torch.bfloat16).view(256, 256)
    h = torch.zeros((256, 256), device=cuda_device)
    pg.precog_block_norm(torch.ones_like(gate), gate=gate, residual=h, residual_out=h, norm="none")
    assert pg.precog_device_status()[0] == 0
    x, got = to_np(gate), to_np(h)
    ref = oracle.silu(x)
    assert np.array_equal(np.isnan(got), np.isnan(x) | np.isneginf(x)) and np.array_equal(np.isposinf(got), np.isposinf(x))
    fine = np.isfinite(x)
    assert fine.sum() > 65_000
    bound = BOUND * np.abs(ref) + np.where(x < -87, 2e-36, 0.0)
    bound += np.where(np.abs(x) < 2.0 ** -100, 2.0 ** -148, 0.0)     # below fp32's normal numbers
    assert float((np.abs(got[fine] - ref[fine]) - bound[fine]).max()) <= 0.0
