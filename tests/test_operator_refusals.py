"""The gated delta rule, head norms and token log probabilities refuse bad arguments on the host:
status codes without any launch, and the binding's own checks (no pointer is dereferenced)."""
import ctypes

import pytest

FAKE = 0x10000  # a 16-byte aligned address that the host never dereferences


@pytest.fixture(scope="module")
def lib():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg.load_library()


def _delta(**kw):
    import paper_2608_02560_gb300 as pg
    s = pg.DeltaInputs(2, 4, 64, 64, pg.PRECOG_BF16, 0.125, FAKE, FAKE, FAKE, FAKE, FAKE, 128, 128, 256)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _scan(lib, s, offsets=FAKE, n=3, T=100, bank=None, bdt=0, entries=0, idx=None, states=FAKE, sdt=0, layer=0, L=1,
          y=None, ydt=0, ws=None, wsb=0):
    return lib.precog_delta_scan(ctypes.byref(s) if s is not None else None, offsets, n, T, bank, bdt, entries, idx,
                                 states, sdt, layer, L, y, ydt, ws, wsb, None)


@pytest.mark.parametrize("change,expect", [
    ({"dk": 12}, 2), ({"dk": 136}, 2), ({"dk": 0}, 2), ({"dv": 4}, 2), ({"dv": 4104}, 2), ({"in_dtype": 2}, 2),
    ({"n_v_heads": 3}, 1), ({"n_qk_heads": 0}, 1), ({"k": 0}, 1), ({"g": 0}, 1), ({"v": FAKE + 8}, 1),
    ({"k_stride": 120}, 1), ({"k_stride": 132}, 1), ({"v_stride": 252}, 1)])
def test_delta_scan_rejects_bad_inputs(lib, change, expect):
    assert _scan(lib, _delta(**change)) == expect
    assert lib.precog_last_error() != b""


@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), 1), (dict(T=1 << 31), 2), (dict(n=-1), 1), (dict(offsets=None), 1), (dict(states=None), 1),
    (dict(sdt=2), 1), (dict(states=FAKE + 4), 1), (dict(layer=1), 1), (dict(layer=-1), 1), (dict(L=0), 1),
    (dict(bank=FAKE, bdt=2, entries=3), 2), (dict(bank=FAKE, entries=2), 1), (dict(bank=FAKE + 2, entries=3), 1),
    (dict(bank=FAKE, entries=-1, idx=FAKE), 1), (dict(idx=FAKE), 1), (dict(y=FAKE, ydt=2), 1), (dict(y=FAKE + 8), 1),
    (dict(n=1 << 40), 2), (dict(n=0), 0)])
def test_delta_scan_rejects_bad_arguments(lib, kw, expect):
    assert _scan(lib, _delta(), **kw) == expect


def test_delta_scan_without_queries_has_no_readout(lib):
    assert _scan(lib, _delta(q=0), y=FAKE) == 1
    assert _scan(lib, None) == 1
    assert lib.precog_delta_scan_workspace_size(None, 1, 1) == 0
    assert lib.precog_delta_scan_workspace_size(ctypes.byref(_delta(dk=4)), 1, 1) == 0


@pytest.mark.parametrize("kw,expect", [
    (dict(n=-1), 1), (dict(states=None), 1), (dict(states=FAKE + 4), 1), (dict(slots_n=2), 1), (dict(slots_n=-1, slots=FAKE), 1),
    (dict(layer=2), 1), (dict(y=None), 1), (dict(ydt=2), 1), (dict(n=0), 0)])
def test_delta_step_rejects_bad_arguments(lib, kw, expect):
    a = dict(n=3, states=FAKE, slots_n=3, slots=None, layer=0, L=2, y=FAKE, ydt=0)
    a.update(kw)
    assert lib.precog_delta_step(ctypes.byref(_delta()), a["n"], a["states"], a["slots_n"], a["slots"], a["layer"], a["L"],
                                 a["y"], a["ydt"], None) == expect
    assert lib.precog_delta_step(ctypes.byref(_delta(q=0)), 3, FAKE, 3, None, 0, 1, FAKE, 0, None) == 1


@pytest.mark.parametrize("kw,expect", [
    ({"dtype": 3}, 2), ({"dim": 260}, 2), ({"dim": 12}, 2), ({"dim": 264}, 2), ({"rot_dim": 3}, 1), ({"rot_dim": 72}, 1),
    ({"norm": 3}, 1), ({"norm": -1}, 1), ({"interleaved": 2}, 1), ({"eps": -1.0}, 1), ({"eps": float("nan")}, 1),
    ({"cos": 0}, 1), ({"sin": FAKE + 2}, 1), ({"d_positions": 0, "n_positions": 9}, 1), ({"n_positions": -1}, 1),
    ({"n_q_heads": -1}, 1), ({"n_k_heads": 1 << 28}, 2), ({"q": 0}, 1), ({"k_out": 0}, 1), ({"q": FAKE + 8}, 1),
    ({"q_weight": FAKE + 4}, 1), ({"q_stride": 120}, 1), ({"k_out_stride": 68}, 1)])
def test_qk_norm_rejects_bad_arguments(lib, kw, expect):
    import paper_2608_02560_gb300 as pg
    a = pg.QkNormArgs(2, 1, 64, 32, pg.PRECOG_BF16, 1, 0, 1e-6, FAKE, FAKE, FAKE, FAKE, 128, 64, 128, 64, None, None,
                      FAKE, FAKE, 100, FAKE)
    for k, v in kw.items():
        setattr(a, k, v)
    assert lib.precog_qk_norm_rope(ctypes.byref(a), 10, None) == expect
    assert lib.precog_qk_norm_rope(None, 10, None) == 1
    assert lib.precog_qk_norm_rope(ctypes.byref(a), -1, None) == 1


def test_qk_norm_of_nothing_launches_nothing(lib):
    import paper_2608_02560_gb300 as pg
    a = pg.QkNormArgs(0, 0, 64, 0, pg.PRECOG_BF16, 1, 0, 1e-6)
    before = lib.precog_launch_count()
    assert lib.precog_qk_norm_rope(ctypes.byref(a), 10, None) == 0
    a.n_q_heads = 2
    assert lib.precog_qk_norm_rope(ctypes.byref(a), 0, None) == 0
    assert lib.precog_launch_count() == before


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=5), 2), (dict(R=-1), 1), (dict(V=0), 1), (dict(V=1 << 30, stride=1 << 30), 2), (dict(stride=99), 1),
    (dict(temp=0.0), 1), (dict(temp=-1.0), 1), (dict(temp=float("nan")), 1), (dict(temp=float("inf")), 1), (dict(temp=1e-45), 1),
    (dict(k=-1), 2), (dict(k=33), 2), (dict(k=20, V=10), 1), (dict(x=None), 1), (dict(x=FAKE + 1), 1), (dict(tok=None), 1),
    (dict(lp=None), 1), (dict(ti=None), 1), (dict(tl=None), 1), (dict(R=0), 0), (dict(R=1 << 31), 2)])
def test_token_logprobs_rejects_bad_arguments(lib, kw, expect):
    a = dict(x=FAKE, dtype=1, R=4, V=100, stride=100, tok=FAKE, temp=1.0, k=2, lp=FAKE, H=None, ti=FAKE, tl=FAKE)
    a.update(kw)
    assert lib.precog_token_logprobs(a["x"], a["dtype"], a["R"], a["V"], a["stride"], a["tok"], a["temp"], a["k"], a["lp"],
                                     a["H"], a["ti"], a["tl"], None) == expect


def test_the_binding_checks_shapes_dtypes_and_devices(lib):
    """Host tensors stand in where the check comes before the pointer is taken."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, v, g = torch.zeros(4, 2, 64), torch.zeros(4, 4, 64), torch.zeros(4, 4)
    with pytest.raises(ValueError, match="GPU"):
        pg.delta_inputs(q, q, v, g, g)
    with pytest.raises(ValueError, match="shapes"):
        pg.delta_inputs(q[:3], q, v, g, g)
    with pytest.raises(TypeError):
        pg.delta_inputs(q, q, v.half(), g, g)
    with pytest.raises(ValueError, match="norm"):
        pg.precog_qk_norm_rope(q, q, q, q, norm="l1")
    with pytest.raises(ValueError, match="shapes"):
        pg.precog_qk_norm_rope(q, q, q[:2], q)
    with pytest.raises(TypeError):
        pg.precog_qk_norm_rope(q, q.half(), q, q)
    with pytest.raises(ValueError, match="together"):
        pg.precog_qk_norm_rope(q, q, q, q, cos=g)
    with pytest.raises(ValueError, match="together"):
        pg.precog_token_logprobs(g, g, g, top_idx=g)
