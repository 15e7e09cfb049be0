"""Entries that are not rotated owe nothing to one another: NaN, infinity and the sign of zero stay with
the entry (and, through the norm, with its head).

Finite outputs are compared as in test_gpu_qk_norm.py."""
import numpy as np
import pytest

import oracle
from tests._util import to_np
from tests.test_gpu_qk_norm import _close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("norm", ["none", "l2", "rms"])
@pytest.mark.parametrize("d,rot,inter,weight", [(64, 0, False, False), (128, 64, False, True), (128, 64, True, False),
                                                (72, 34, True, False), (256, 8, False, False), (40, 2, True, True)])
def test_broken_entries_beyond_the_rotation(cuda_device, dtype, norm, d, rot, inter, weight):
    import torch
    import paper_2608_02560_gb300 as pg
    T, h = 9, 3
    gen = torch.Generator(device=cuda_device).manual_seed(d + rot)
    x = torch.randn((T, h, d), device=cuda_device, generator=gen).to(getattr(torch, dtype))
    x[0, 0, rot:] = -0.0
    x[1, 1, d - 1] = float("inf")
    x[2, 0, rot] = float("-inf")
    x[3, 2, d - 2] = float("nan")
    if rot:
        x[4, 0, 0] = float("inf")
    w = torch.randn(d, device=cuda_device, generator=gen) if weight else None
    ang = torch.rand((T, rot // 2), device=cuda_device, generator=gen) * 10
    cos, sin = (torch.cos(ang), torch.sin(ang)) if rot else (None, None)
    out, none = torch.empty_like(x), torch.empty((T, 0, d), dtype=x.dtype, device=cuda_device)
    pg.precog_qk_norm_rope(x, none, out, none, norm=norm, q_weight=w, cos=cos, sin=sin, interleaved=inter)
    n = lambda t: None if t is None else to_np(t)  # noqa: E731
    with np.errstate(invalid="ignore", over="ignore"):
        ref = oracle.qk_norm_rope(n(x), norm, 1e-6, n(w), n(cos), n(sin), None, inter)
    got = to_np(out)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref))
    fine = np.isfinite(ref).all(-1)
    _close(out[torch.from_numpy(fine)], ref[fine])
    if norm == "none" and not weight:
        assert torch.equal(torch.signbit(out[..., rot:]) | torch.isnan(out[..., rot:]),
                           torch.signbit(x[..., rot:]) | torch.isnan(x[..., rot:]))
