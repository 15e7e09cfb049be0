"""Norms of query and key heads with the rotation against the fp64 definition.

Tolerance: each output is a sum of two products of values with a handful of fp32 roundings, so
it lies within 16 * 2^-24 of the vector's largest magnitude, and its own rounding to 16 bits."""
import numpy as np
import pytest

import oracle
from tests._util import to_np

pytestmark = pytest.mark.gpu


def _close(got, ref):
    import torch
    scale = np.max(np.abs(ref), axis=-1, keepdims=True) + 1e-30
    unit = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[got.dtype]
    floor = 2.0 ** -25 if got.dtype == torch.float16 else 0.0      # half an fp16 subnormal step
    lim = 2 * 16 * 2.0 ** -24 * scale + unit * np.abs(ref) + floor
    assert np.all(np.abs(to_np(got) - ref) <= lim), float(np.max(np.abs(to_np(got) - ref) / lim))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("T,hq,hk,d,rot,norm,inter,weight", [
    (1, 16, 8, 128, 64, "l2", False, False), (37, 4, 2, 128, 128, "rms", True, True),
    (5, 3, 1, 8, 8, "l2", False, True), (300, 2, 2, 256, 256, "rms", False, True),
    (11, 1, 0, 72, 34, "l2", False, False), (11, 0, 5, 72, 34, "rms", True, True),
    (9, 7, 3, 40, 0, "l2", False, True), (64, 2, 1, 64, 24, "none", False, False),
    (3, 1, 1, 248, 246, "none", True, True), (1000, 5, 5, 96, 48, "rms", False, False)])
def test_matches_the_definition(cuda_device, dtype, T, hq, hk, d, rot, norm, inter, weight):
    import torch
    import paper_2608_02560_gb300 as pg
    dt = getattr(torch, dtype)
    gen = torch.Generator(device=cuda_device).manual_seed(T + d + rot)
    proj = torch.randn((T, (hq + 2 * hk) * d + 8), device=cuda_device, generator=gen).to(dt)
    q, k = proj[:, :hq * d].view(T, hq, d), proj[:, hq * d:(hq + hk) * d].view(T, hk, d)
    wq, wk = (torch.randn((2, d), device=cuda_device, generator=gen) if weight else (None, None))
    n_pos = 50
    ang = torch.rand((n_pos, rot // 2), device=cuda_device, generator=gen) * 100
    cos, sin = (torch.cos(ang), torch.sin(ang)) if rot else (None, None)
    pos = torch.randint(0, n_pos, (T,), device=cuda_device, generator=gen)
    qo, ko = (torch.full((T, h, d), float("nan"), dtype=dt, device=cuda_device) for h in (hq, hk))
    pg.precog_qk_norm_rope(q, k, qo, ko, norm=norm, q_weight=wq, k_weight=wk, eps=1e-6, cos=cos, sin=sin,
                           positions=pos if rot else None, interleaved=inter)
    n = lambda t: None if t is None else to_np(t)  # noqa: E731
    for x, w, out in ((q, wq, qo), (k, wk, ko)):
        if x.shape[1]:
            _close(out, oracle.qk_norm_rope(n(x), norm, 1e-6, n(w), n(cos), n(sin), n(pos).astype(int), inter))
    # in place
    pg.precog_qk_norm_rope(q, k, q, k, norm=norm, q_weight=wq, k_weight=wk, eps=1e-6, cos=cos, sin=sin,
                           positions=pos if rot else None, interleaved=inter)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert pg.precog_device_status()[0] == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("hq,hk,d,rot,inter,weight", [(9, 10, 72, 48, False, True), (17, 1, 64, 30, True, False),
                                                      (3, 12, 200, 200, False, False)])
def test_many_tokens(cuda_device, dtype, hq, hk, d, rot, inter, weight):
    """Enough tokens for groups of eight heads, whose last group has fewer."""
    import torch
    import paper_2608_02560_gb300 as pg
    T, n_pos, dt = 6001, 300, getattr(torch, dtype)
    gen = torch.Generator(device=cuda_device).manual_seed(d)
    proj = torch.randn((T, (hq + hk) * d), device=cuda_device, generator=gen).to(dt)
    q, k = proj[:, :hq * d].view(T, hq, d), proj[:, hq * d:].view(T, hk, d)
    wq, wk = (torch.randn((2, d), device=cuda_device, generator=gen) if weight else (None, None))
    ang = torch.rand((n_pos, rot // 2), device=cuda_device, generator=gen) * 100
    cos, sin = torch.cos(ang), torch.sin(ang)
    pos = torch.randint(0, n_pos, (T,), device=cuda_device, generator=gen)
    qo, ko = (torch.full((T, h, d), float("nan"), dtype=dt, device=cuda_device) for h in (hq, hk))
    pg.precog_qk_norm_rope(q, k, qo, ko, norm="rms", q_weight=wq, k_weight=wk, cos=cos, sin=sin, positions=pos,
                           interleaved=inter)
    n = lambda t: None if t is None else to_np(t)  # noqa: E731
    for x, w, out in ((q, wq, qo), (k, wk, ko)):
        _close(out, oracle.qk_norm_rope(n(x), "rms", 1e-6, n(w), n(cos), n(sin), n(pos).astype(int), inter))


def test_zero_vectors_extremes_and_default_positions(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    x = torch.zeros((4, 1, 64), device=cuda_device)
    x[1] = 1e-18
    x[2] = 1e18
    x[3, 0, 5] = float("nan")
    ang = torch.arange(4, device=cuda_device)[:, None] * torch.ones(32, device=cuda_device)
    out, none = torch.empty_like(x), torch.empty((4, 0, 64), device=cuda_device)
    pg.precog_qk_norm_rope(x, none, out, none, norm="l2", eps=1e-6, cos=torch.cos(ang), sin=torch.sin(ang))
    ref = oracle.qk_norm_rope(to_np(x[:3]), "l2", 1e-6, None, to_np(torch.cos(ang)), to_np(torch.sin(ang)))
    _close(out[:3], ref)
    assert bool(torch.isnan(out[3]).all()) and bool((out[0] == 0).all())


def test_positions_outside_the_table(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    q = torch.randn((3, 2, 64), device=cuda_device)
    out, none = torch.full_like(q, 7.0), torch.empty((3, 0, 64), device=cuda_device)
    cos, sin = torch.ones((5, 32), device=cuda_device), torch.zeros((5, 32), device=cuda_device)
    pg.precog_qk_norm_rope(q, none, out, none, norm="none", cos=cos, sin=sin,
                           positions=torch.tensor([5, 4, -1], device=cuda_device))
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    assert bool((out[0] == 7).all()) and bool((out[2] == 7).all()) and torch.equal(out[1], q[1])


def test_rows_past_32_bits(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    T, stride = 200, 2 ** 24
    wide = torch.zeros((T - 1) * stride + 256, dtype=torch.bfloat16, device=cuda_device)
    q = wide.as_strided((T, 2, 128), (stride, 128, 1))
    src = torch.randn((T, 2, 128), device=cuda_device).to(torch.bfloat16)
    q.copy_(src)
    none = torch.empty((T, 0, 128), dtype=torch.bfloat16, device=cuda_device)
    out, ref = torch.empty_like(src), torch.empty_like(src)
    pg.precog_qk_norm_rope(q, none, out, none)
    pg.precog_qk_norm_rope(src, none, ref, none)
    assert torch.equal(out, ref)
