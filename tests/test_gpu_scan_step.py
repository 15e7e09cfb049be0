"""Single tokens of the diagonal scan on a table of states, against the fp64 definition (bounds: tests/_layer.py)
and against the framework's own scan of the same tokens."""
import numpy as np
import pytest

import oracle
from tests._layer import close, step_bound
from tests._util import TOL_F32, rel_err, to_np

pytestmark = pytest.mark.gpu
N = 16


def _case(dev, L, n, D, dtype, cplx, seed, slots=None, layers=None, growth=0.0):
    import torch
    gen = torch.Generator(device=dev).manual_seed(seed)
    rn = lambda *s: torch.randn(s, device=dev, generator=gen)  # noqa: E731
    x, dt = rn(L, n, D).to(dtype), torch.nn.functional.softplus(rn(L, n, D) - 1).to(dtype)
    B, C = rn(L, n, N).to(dtype), rn(L, n, N).to(dtype)
    A = -torch.exp(rn(L, D, N)) + growth
    h = rn(slots or n, layers or L, D, N)
    if cplx:
        A, h = torch.complex(A, 40.0 * rn(L, D, N)), torch.complex(h, rn(slots or n, layers or L, D, N))
    return x, dt, B, C, A, h, rn


def _np(t):
    return t.detach().cpu().numpy().astype(np.complex128) if t.is_complex() else to_np(t)


def _check(got_h, got_y, x, dt, A, B, C, h0, skip, gate):
    a = [_np(t) for t in (x, dt, A, B, C, h0)]
    s, g = (None if t is None else _np(t) for t in (skip, gate))
    h, y = oracle.scan_step(*a, skip=s, gate=g)
    state, out = step_bound(a[0], a[1], a[2], a[3], a[4], a[5], h, y, s, g, x.dtype)
    got = _np(got_h)
    if np.iscomplexobj(h):
        close(got.real, h.real, state, "float32")
        close(got.imag, h.imag, state, "float32")
    else:
        close(got, h, state, "float32")
    close(_np(got_y), y, out, got_y.dtype)


@pytest.mark.parametrize("dtype,y_dtype", [("bfloat16", "bfloat16"), ("float32", "float32"), ("bfloat16", "float32")])
@pytest.mark.parametrize("cplx", [False, True])
@pytest.mark.parametrize("L,n,D,skip,gate", [(1, 1, 8, False, False), (24, 1, 256, True, True), (3, 5, 72, True, False),
                                             (2, 67, 264, False, True), (1, 300, 1032, True, True)])
def test_steps_match_the_definition(cuda_device, dtype, y_dtype, cplx, L, n, D, skip, gate):
    import torch
    import paper_2608_02560_gb300 as pg
    d, dt_ = cuda_device, getattr(torch, dtype)
    x, dt, B, C, A, h, rn = _case(d, L, n, D, dt_, cplx, 11 + n, slots=n + 7, layers=L + 2)
    slots = torch.randperm(n + 7, device=d)[:n].contiguous()
    if n > 1:
        slots[n // 2] = -1
    s = rn(L, D) if skip else None
    g = rn(n, L, D + 8).to(dt_).transpose(0, 1)[:, :, 8:] if gate else None     # strided rows and layers
    before = h.clone()
    y = torch.full((L, n, D), 9.0, dtype=getattr(torch, y_dtype), device=d)
    kind = pg.PRECOG_A_COMPLEX if cplx else pg.PRECOG_A_GENERAL
    pg.precog_scan_step(pg.scan_inputs(x, dt, B, A, C, a_kind=kind), h, slots=slots, layer0=1, skip=s, gate=g, y_out=y)
    assert pg.precog_device_status()[0] == 0
    live = slots >= 0
    rows = slots[live]
    for l in range(L):
        _check(h[rows, 1 + l], y[l][live], x[l][live], dt[l][live], A[l], B[l][live], C[l][live], before[rows, 1 + l],
               None if s is None else s[l], None if g is None else g[l][live])
    assert bool((y[:, ~live] == 0).all())
    h[rows, 1:1 + L] = before[rows, 1:1 + L]
    assert torch.equal(h, before)                       # other layers and slots are untouched


@pytest.mark.parametrize("cplx", [False, True])
def test_tokens_one_by_one_are_the_scan(cuda_device, cplx):
    """Prefill of 40 tokens from injected states against 40 steps: both within TOL_F32 of the recurrence."""
    import torch
    import paper_2608_02560_gb300 as pg
    d, L, n, D, T = cuda_device, 2, 3, 64, 40
    x, dt, B, C, A, h, _ = _case(d, L, n * T, D, torch.float32, cplx, 5, slots=n)
    if cplx:   # the scan's own range of angles
        A = torch.complex(A.real.contiguous(), (np.pi * torch.arange(N, device=d)).expand(L, D, N).contiguous())
    kind = pg.PRECOG_A_COMPLEX if cplx else pg.PRECOG_A_GENERAL
    y, behind = torch.empty((L, n * T, D), device=d), torch.empty_like(h)
    pg.precog_prefill_from_state(pg.scan_inputs(x, dt, B, A, C, a_kind=kind), n, T, h, y_out=y, state_out=behind)
    got = torch.empty_like(y)
    for t in range(T):
        rows = torch.arange(n, device=d) * T + t
        step = torch.empty((L, n, D), device=d)
        pg.precog_scan_step(pg.scan_inputs(*(v[:, rows].contiguous() for v in (x, dt, B)), A, C[:, rows].contiguous(),
                                           a_kind=kind), h, y_out=step)
        got[:, rows] = step
    assert pg.precog_device_status()[0] == 0
    assert rel_err(to_np(got), to_np(y)) < 2 * TOL_F32
    real = torch.view_as_real if cplx else (lambda t: t)
    assert rel_err(to_np(real(h)), to_np(real(behind))) < 2 * TOL_F32


def test_growth_beyond_fp32_and_broken_rows(cuda_device):
    """e^(dt A) may leave fp32 where the state is zero or tiny; NaN in one row or channel touches no other."""
    import torch
    import paper_2608_02560_gb300 as pg
    d = cuda_device
    x, dt, B, C, A, h, _ = _case(d, 1, 4, 64, torch.float32, False, 7)
    A[0, 5], dt[0, 0, 5] = 60.0, 2.0            # e^120
    h[0, 0, 5] = 0.0
    h[0, 0, 5, 3] = 1e-20
    x[0, 1, 9] = float("nan")
    B[0, 2, 1] = float("inf")
    before = h.clone()
    y = torch.empty((1, 4, 64), device=d)
    pg.precog_scan_step(pg.scan_inputs(x, dt, B, A, C), h, y_out=y)
    with np.errstate(invalid="ignore"):
        ref, ref_y = oracle.scan_step(*(to_np(t[0]) for t in (x, dt, A, B, C)), to_np(before[:, 0]))
    assert np.array_equal(np.isfinite(to_np(h[:, 0])), np.isfinite(ref))
    assert np.array_equal(np.isfinite(to_np(y[0])), np.isfinite(ref_y))
    assert np.isnan(to_np(h[1, 0, 9])).all() and not np.isfinite(to_np(y[0, 2])).any()
    for i in (0, 3):
        _check(h[i:i + 1, 0], y[0, i:i + 1], x[0, i:i + 1], dt[0, i:i + 1], A[0], B[0, i:i + 1], C[0, i:i + 1],
               before[i:i + 1, 0], None, None)


def test_slots_outside_the_table_are_idle_and_flagged(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    d = cuda_device
    x, dt, B, C, A, h, _ = _case(d, 2, 4, 64, torch.float32, False, 9)
    before, y = h.clone(), torch.full((2, 4, 64), 9.0, device=d)
    pg.precog_scan_step(pg.scan_inputs(x, dt, B, A, C), h, slots=torch.tensor([4, -2, -(1 << 40), 1], device=d), y_out=y)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    assert bool((y[:, :3] == 0).all()) and bool((y[:, 3] != 9.0).all())
    assert torch.equal(h[[0, 2, 3]], before[[0, 2, 3]]) and bool((h[1] != before[1]).any())


def test_offsets_beyond_32_bits(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    d, slots, D = cuda_device, 33_000, 8200
    h = torch.zeros((slots, 1, D, N), device=d)
    assert h.numel() > 1 << 32
    x, dt, B, C, A, small, _ = _case(d, 1, 2, D, torch.bfloat16, False, 3)
    where = torch.tensor([slots - 1, 0], dtype=torch.int64, device=d)
    h[where] = small
    y = torch.empty((1, 2, D), device=d)
    pg.precog_scan_step(pg.scan_inputs(x, dt, B, A, C), h, slots=where, y_out=y)
    assert pg.precog_device_status()[0] == 0
    _check(h[where, 0], y[0], x[0], dt[0], A[0], B[0], C[0], small[:, 0], None, None)
    assert not bool(h[1:-1].any())
