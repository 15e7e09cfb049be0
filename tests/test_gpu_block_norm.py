"""Skip, gate, norm and residual at the end of a block against the fp64 definition (bounds: tests/_layer.py)."""
import itertools

import numpy as np
import pytest

import oracle
from tests._layer import close, norm_bound
from tests._util import to_np

pytestmark = pytest.mark.gpu


def _run(dev, T, D, dtype, res=None, skip=False, gate=None, weight=True, norm=True, groups=1, scale=1.0, out=True, pad=0,
         seed=0, mend=None, eps=1e-6, inplace=False):
    """One call and its check; ``mend`` changes the inputs first."""
    import torch
    import paper_2608_02560_gb300 as pg
    gen = torch.Generator(device=dev).manual_seed(seed + 31 * T + D)
    rn = lambda *s: torch.randn(s, device=dev, generator=gen)  # noqa: E731
    dt = getattr(torch, dtype)
    rows = lambda t: rn(T, D + pad).to(t)[:, pad // 2:pad // 2 + D]  # noqa: E731
    t = dict(x=rows(dt), skip=rn(D) if skip else None, skip_input=rows(dt) if skip else None,
             gate=rows(dt) if gate else None, weight=1 + 0.3 * rn(D) if norm and weight else None,
             residual=3 * rows(getattr(torch, res)) if res else None,
             out_weight=1 + 0.3 * rn(D) if res and out and weight else None)
    s = 0.5 * rn(D) if scale == "vector" else scale
    if mend:
        mend(t)
    args = {k: None if v is None else to_np(v) for k, v in t.items()}
    args.update(groups=groups, norm=norm, gate_first=gate == "before", scale=to_np(s) if scale == "vector" else s,
                out_norm=bool(res and out), eps=eps)
    with np.errstate(invalid="ignore", over="ignore"):
        ref, ref_h = oracle.block_norm(**args)
        args.pop("eps")
        bound, bound_h = norm_bound(args, dt, eps)
    wide = torch.full((T + 2, D + pad), 7.0, dtype=dt, device=dev)
    o = (wide[1:-1, pad // 2:pad // 2 + D] if not inplace else t["x"]) if out else None
    h = None
    if res:
        h = t["residual"] if inplace else torch.full((T, D), 9.0, dtype=t["residual"].dtype, device=dev)
    pg.precog_block_norm(t["x"], out=o, skip=t["skip"], skip_input=t["skip_input"], gate=t["gate"],
                         gate_first=gate == "before", weight=t["weight"], groups=groups, residual=t["residual"], scale=s,
                         residual_out=h, out_weight=t["out_weight"], eps=eps, norm="rms" if norm else "none")
    assert pg.precog_device_status()[0] == 0
    if out:
        close(to_np(o), ref, np.nan_to_num(bound), dt)
        if not inplace:
            o.fill_(7.0)
            assert bool((wide == 7.0).all())            # nothing beside the rows
    if res:
        close(to_np(h), ref_h, np.nan_to_num(bound_h), h.dtype)
    return ref, ref_h


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,D", [(1, 8), (3, 16), (1, 2048), (5, 248), (9, 264), (17, 520), (4, 1032), (33, 2056), (3, 4096),
                                 (5, 4104), (2, 8192), (3, 8200), (2, 16384)])
def test_a_norm_of_rows(cuda_device, dtype, T, D):
    _run(cuda_device, T, D, dtype, pad=16)


FORMS = [f for f in itertools.product([None, "float32", "bfloat16"], [False, True], [None, "before", "after"], [False, True],
                                      [1.0, 0.7, "vector"], [False, True])
         if (f[0] or f[5]) and (f[0] or f[4] == 1.0)]


@pytest.mark.parametrize("res,skip,gate,norm,scale,out", FORMS)
def test_every_form(cuda_device, res, skip, gate, norm, scale, out):
    for dtype in ("bfloat16",) if res == "bfloat16" else ("bfloat16", "float32"):
        for T, D in ((7, 200), (3, 1096)):
            _run(cuda_device, T, D, dtype, res, skip, gate, True, norm, 1, scale, out, pad=16)


@pytest.mark.parametrize("groups,D", [(2, 16), (4, 1024), (8, 2048), (64, 4096), (3, 24 * 41), (2, 32768), (128, 65536)])
def test_groups(cuda_device, groups, D):
    for dtype in ("bfloat16", "float32"):
        _run(cuda_device, 5, D, dtype, skip=True, gate="before", groups=groups, pad=16)
        _run(cuda_device, 2, D, dtype, res="float32", gate="after", groups=groups, out=False)


@pytest.mark.parametrize("res", [None, "float32", "bfloat16"])
def test_in_place_and_without_weights(cuda_device, res):
    _run(cuda_device, 19, 776, "bfloat16", res, True, "before", False, True, 1, 0.5 if res else 1.0, True, pad=32, inplace=True)


def test_no_rows_of_zero_eps_and_many_rows(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    x = torch.empty((0, 64), device=cuda_device)
    before = pg.precog_launch_count()
    pg.precog_block_norm(x, out=torch.empty_like(x))
    assert pg.precog_launch_count() == before
    _run(cuda_device, 6, 64, "float32", eps=0.0)
    _run(cuda_device, 30_001, 72, "bfloat16", res="float32", gate="after")


@pytest.mark.parametrize("what", ["zero", "nan", "inf", "gate-inf", "large", "masked"])
def test_rows_that_break_break_alone(cuda_device, what):
    def mend(t):
        if what == "zero":
            t["x"][2], t["skip_input"][2] = 0.0, 0.0
        elif what == "nan":
            t["x"][1, 5] = float("nan")
            t["residual"][3, 7] = float("nan")
        elif what == "inf":
            t["x"][1, 5], t["residual"][2, 9] = float("inf"), float("-inf")
        elif what == "gate-inf":
            t["gate"][1, 0], t["gate"][2, 1] = float("-inf"), float("inf")
        elif what == "large":
            t["x"][1] *= 2.0 ** 50
            t["residual"][4] *= 2.0 ** 40
        elif what == "masked":
            t["gate"][0] = -200.0
    ref, h = _run(cuda_device, 6, 136, "float32", "float32", True, "before", mend=mend)
    if what in ("zero", "large", "masked"):
        assert np.isfinite(ref).all() and np.isfinite(h).all()
    else:
        assert np.isfinite(ref[[0, 5]]).all() and not np.isfinite(ref).all()
