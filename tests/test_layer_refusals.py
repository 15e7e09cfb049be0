"""The causal convolution, the scan's single tokens, the block norm and the adjusted logits refuse bad arguments
on the host: status codes without any launch, and the binding's own checks (no pointer is dereferenced)."""
import ctypes

import pytest

FAKE = 0x10000000  # a 16-byte aligned address that the host never dereferences
X, Y, W, T1, T2 = (FAKE + i * 0x1000000 for i in range(5))   # 16 MiB apart


@pytest.fixture(scope="module")
def lib():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg.load_library()


def _set(s, kw):
    for k, v in kw.items():
        assert k in dict(s._fields_)
        setattr(s, k, v)
    return s


def _conv_args(**kw):
    import paper_2608_02560_gb300 as pg
    return _set(pg.ConvArgs(pg.PRECOG_BF16, 64, 4, 1, X, Y, 64, 64, W, None), kw)


def _conv(lib, s, offsets=W, n=3, T=100, bank=None, entries=0, idx=None, out=T1, layer=0, L=1):
    return lib.precog_causal_conv(ctypes.byref(s) if s is not None else None, offsets, n, T, bank, entries, idx, out, layer,
                                  L, None)


def _conv_step(lib, s, n=3, windows=T1, n_slots=3, slots=None, layer=0, L=1):
    return lib.precog_conv_step(ctypes.byref(s) if s is not None else None, n, windows, n_slots, slots, layer, L, None)


@pytest.mark.parametrize("change,expect", [
    ({"dtype": 2}, 2), ({"dtype": 7}, 2), ({"dim": 0}, 2), ({"dim": 12}, 2), ({"dim": -8}, 2), ({"kernel": 1}, 2),
    ({"kernel": 5}, 2), ({"silu": 2}, 1), ({"x": 0}, 1), ({"y": 0}, 1), ({"x": X + 8}, 1), ({"y": Y + 2}, 1),
    ({"weight": 0}, 1), ({"weight": W + 4}, 1), ({"bias": W + 4}, 1), ({"x_stride": 56}, 1), ({"y_stride": 68}, 1),
    ({"x_stride": -64}, 1), ({"y": X + 128}, 1)])
def test_convolutions_reject_bad_rows(lib, change, expect):
    assert _conv(lib, _conv_args(**change)) == expect
    assert lib.precog_last_error() != b""
    assert _conv_step(lib, _conv_args(**change)) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), 1), (dict(T=1 << 31), 2), (dict(n=-1), 1), (dict(n=1 << 30, out=None), 2), (dict(offsets=None), 1),
    (dict(offsets=W + 4), 1), (dict(bank=T2, entries=3, idx=W + 4), 1),
    (dict(layer=1), 1), (dict(layer=-1), 1), (dict(L=0), 1), (dict(out=T1 + 8), 1), (dict(bank=T2 + 8, entries=3), 1),
    (dict(bank=T2, entries=2), 1), (dict(bank=T2, entries=-1, idx=W), 1), (dict(bank=T1, entries=3), 1),
    (dict(bank=T1 + 384, entries=3), 1), (dict(out=X), 1), (dict(out=Y + 64), 1), (dict(bank=Y, entries=3), 1),
    (dict(n=1 << 30, L=1 << 30), 2), (dict(n=0), 0), (dict(n=0, T=0, out=None), 0)])
def test_causal_conv_rejects_bad_arguments(lib, kw, expect):
    before = lib.precog_launch_count()
    assert _conv(lib, _conv_args(), **kw) == expect
    assert _conv(lib, None) == 1
    assert lib.precog_launch_count() == before


def test_causal_conv_does_not_run_in_place_and_takes_slices(lib):
    assert _conv(lib, _conv_args(y=X)) == 1
    assert _conv(lib, _conv_args(y=X + 128, x_stride=128, y_stride=128), n=0) == 0       # halves of one buffer
    assert _conv(lib, _conv_args(y=X + 112, x_stride=128, y_stride=128), n=0) == 1
    assert _conv(lib, _conv_args(y=X + 128, x_stride=128, y_stride=64), n=0) == 1


@pytest.mark.parametrize("kw,expect", [
    (dict(n=-1), 1), (dict(slots=W + 4), 1), (dict(windows=None), 1), (dict(windows=T1 + 8), 1), (dict(n_slots=2), 1), (dict(n_slots=-1, slots=W), 1),
    (dict(layer=1), 1), (dict(L=0), 1), (dict(windows=X), 1), (dict(windows=Y + 128), 1), (dict(n=1 << 31, slots=W, L=1), 2),
    (dict(n_slots=1 << 62, slots=W), 2), (dict(n=0, n_slots=0), 0)])
def test_conv_step_rejects_bad_arguments(lib, kw, expect):
    assert _conv_step(lib, _conv_args(), **kw) == expect
    assert _conv_step(lib, None) == 1


def _scan_step(lib, n=3, states=T1, n_slots=3, slots=None, layer0=0, L=2, skip=None, gate=None, gs=64, gls=192, y=Y, ydt=0,
               reserved=0, **change):
    import paper_2608_02560_gb300 as pg
    s = _set(pg.ScanInputs(2, 64, 16, pg.PRECOG_BF16, pg.PRECOG_A_GENERAL, 0, X, X + 0x10000, X + 0x20000, X + 0x30000,
                           X + 0x40000, 192, 48), change)
    a = pg.ScanStepArgs(states, n_slots, slots, layer0, L, skip, gate, gs, gls, y, ydt, reserved)
    return lib.precog_scan_step(ctypes.byref(s), ctypes.byref(a), n, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(reserved=1), 1), (dict(N=8), 2), (dict(D=12), 2), (dict(in_dtype=2), 2), (dict(a_kind=3), 1), (dict(x=0), 1), (dict(C=0), 1), (dict(A=0), 1),
    (dict(layer_stride_xd=128), 1), (dict(n=-1), 1), (dict(n=1 << 31), 2), (dict(states=None), 1), (dict(states=T1 + 8), 1),
    (dict(n_slots=2), 1), (dict(slots=W + 4), 1), (dict(n_slots=-1, slots=W), 1), (dict(layer0=1), 1), (dict(layer0=-1), 1), (dict(L=1), 1),
    (dict(y=None), 1), (dict(y=Y + 8), 1), (dict(ydt=2), 1), (dict(skip=W + 4), 1), (dict(gate=W + 8), 1), (dict(gate=W, gs=56), 1),
    (dict(gate=W, gs=68), 1), (dict(gate=W, gls=60), 1), (dict(gate=W, gls=196), 1), (dict(y=X), 1), (dict(y=T1 + 512), 1),
    (dict(states=X), 1), (dict(gate=Y), 1), (dict(gate=T1), 1), (dict(gate=Y - 256, gs=64, gls=192), 1),
    (dict(n_slots=1 << 60, slots=W), 2), (dict(n=0, n_slots=0, x=0, dt=0, B=0, C=0), 0)])
def test_scan_step_rejects_bad_arguments(lib, kw, expect):
    before = lib.precog_launch_count()
    assert _scan_step(lib, **kw) == expect
    assert lib.precog_launch_count() == before
    import paper_2608_02560_gb300 as pg
    assert lib.precog_scan_step(None, ctypes.byref(pg.ScanStepArgs(T1, 1, None, 0, 1, None, None, 0, 0, Y, 0, 0)), 1, None) == 1
    assert lib.precog_scan_step(ctypes.byref(pg.ScanInputs()), None, 1, None) == 1


def _norm_args(**kw):
    import paper_2608_02560_gb300 as pg
    return _set(pg.BlockNormArgs(pg.PRECOG_BF16, pg.PRECOG_F32, 64, 1, pg.PRECOG_NORM_RMS, 1, 1.0, 1e-6, X, None, None, T1,
                                 T1, Y, 64, 64, 64, 64, 64, 64), kw)


@pytest.mark.parametrize("change,expect", [
    ({"dtype": 2}, 2), ({"residual_dtype": 2}, 2), ({"dtype": 0, "residual_dtype": 1}, 2), ({"dim": 0}, 1), ({"dim": 60}, 2),
    ({"groups": 0}, 1), ({"groups": 16, "residual": 0, "residual_out": 0}, 2), ({"groups": 2}, 2), ({"dim": 16392}, 2),
    ({"norm": 1}, 1), ({"norm": 3}, 1), ({"gate_first": 2}, 1), ({"eps": -1e-6}, 1), ({"eps": float("nan")}, 1), ({"x": 0}, 1),
    ({"skip": W}, 1), ({"skip_input": W}, 1), ({"residual": 0}, 1), ({"residual_out": 0}, 1),
    ({"residual": 0, "residual_out": 0, "out": 0}, 1), ({"x": X + 8}, 1), ({"out": Y + 4}, 1), ({"x_stride": 56}, 1),
    ({"gate": W, "gate_stride": 68}, 1), ({"weight": W + 4}, 1), ({"out_weight": W + 8}, 1), ({"scale_weight": W + 2}, 1),
    ({"out": X + 128}, 1), ({"out": T1}, 1), ({"residual_out": X}, 1), ({"residual_out": T1 + 256}, 1),
    ({"residual_dtype": 1, "residual_out": Y}, 1), ({"gate": Y + 16}, 1), ({"weight": Y + 256}, 1), ({"out_weight": T1 + 64}, 1),
    ({"scale_weight": Y}, 1)])
def test_block_norm_rejects_bad_arguments(lib, change, expect):
    assert lib.precog_block_norm(ctypes.byref(_norm_args(**change)), 10, None) == expect
    assert lib.precog_last_error() != b""


def test_block_norm_of_nothing_launches_nothing(lib):
    before = lib.precog_launch_count()
    assert lib.precog_block_norm(None, 10, None) == 1
    assert lib.precog_block_norm(ctypes.byref(_norm_args()), -1, None) == 1
    assert lib.precog_block_norm(ctypes.byref(_norm_args()), 0, None) == 0
    assert lib.precog_block_norm(ctypes.byref(_norm_args(x=0, out=0, residual=0, residual_out=0)), 0, None) == 0
    assert lib.precog_block_norm(ctypes.byref(_norm_args(residual=0, residual_out=0)), 1 << 31, None) == 2
    assert lib.precog_launch_count() == before


def _adjust_args(**kw):
    import paper_2608_02560_gb300 as pg
    a = pg.AdjustArgs(dtype=pg.PRECOG_BF16, vocab=100, stride=100, out_stride=100, logits=X, out=Y, d_history=W,
                      d_history_offsets=W, n_history=50, d_repetition=W, d_bias_idx=W, d_bias=W, d_bias_offsets=W, n_bias=9,
                      d_mask=W, n_masks=4)
    return _set(a, kw)


@pytest.mark.parametrize("change,expect", [
    ({"dtype": 3}, 2), ({"reserved": 1}, 1), ({"vocab": 0}, 1), ({"vocab": 1 << 30, "stride": 1 << 30, "out_stride": 1 << 30}, 2),
    ({"stride": 99}, 1), ({"out_stride": -1}, 1), ({"n_history": -1}, 1), ({"n_bias": -1}, 1), ({"n_masks": -1}, 1),
    ({"n_history": 1 << 30}, 2), ({"n_bias": 1 << 30}, 2), ({"logits": 0}, 1), ({"out": 0}, 1), ({"logits": X + 1}, 1),
    ({"out": Y + 1}, 1), ({"out": X + 2}, 1), ({"d_history": 0}, 1), ({"d_history_offsets": 0}, 1), ({"d_bias": 0}, 1),
    ({"d_bias_idx": 0}, 1), ({"d_bias_offsets": 0}, 1), ({"n_masks": 3}, 1), ({"d_mask": 0, "d_mask_rows": W}, 1),
    ({"d_history": W + 4}, 1), ({"d_history_offsets": W + 4}, 1), ({"d_count_from": W + 4}, 1), ({"d_bias_idx": W + 4}, 1),
    ({"d_bias_offsets": W + 4}, 1), ({"d_mask_rows": W + 4}, 1), ({"d_repetition": W + 2}, 1), ({"d_frequency": W + 1}, 1),
    ({"d_presence": W + 2}, 1), ({"d_bias": W + 2}, 1), ({"d_mask": W + 2}, 1)])
def test_adjust_logits_rejects_bad_arguments(lib, change, expect):
    assert lib.precog_adjust_logits(ctypes.byref(_adjust_args(**change)), 4, None) == expect
    assert lib.precog_last_error() != b""


def test_adjust_logits_of_nothing_launches_nothing(lib):
    before = lib.precog_launch_count()
    assert lib.precog_adjust_logits(None, 4, None) == 1
    assert lib.precog_adjust_logits(ctypes.byref(_adjust_args()), -1, None) == 1
    assert lib.precog_adjust_logits(ctypes.byref(_adjust_args()), 0, None) == 0
    assert lib.precog_adjust_logits(ctypes.byref(_adjust_args(d_mask=0, n_masks=0, out=T1, out_stride=1 << 40, stride=1 << 40)),
                                    1 << 40, None) == 2
    assert lib.precog_launch_count() == before


def test_the_binding_checks_shapes_dtypes_and_devices(lib, monkeypatch):
    """Host tensors stand in where the check comes before the pointer is taken."""
    import torch
    import paper_2608_02560_gb300 as pg
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    x, w, off = torch.zeros(6, 8), torch.zeros(8, 4), torch.zeros(3, dtype=torch.int64)
    win, g = torch.zeros(2, 1, 3, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError, match="y_out"):
        pg.precog_causal_conv(x, w, off)
    with pytest.raises(ValueError, match="y_out"):
        pg.precog_causal_conv(x, w, off, y_out=x[:3])
    with pytest.raises(ValueError, match="without bank"):
        pg.precog_causal_conv(x, w, off, idx=off, y_out=g)
    with pytest.raises(ValueError, match="bank must be"):
        pg.precog_causal_conv(x, w, off, bank=win[:, :, :2], y_out=g)
    with pytest.raises(ValueError, match="one entry per sequence"):
        pg.precog_causal_conv(x, w, off, windows_out=win[:1], y_out=g)
    with pytest.raises(ValueError, match="number of layers"):
        pg.precog_causal_conv(x, w, off, bank=win.repeat(1, 2, 1, 1), windows_out=win, y_out=g)
    with pytest.raises(ValueError, match="rows of x"):
        pg.precog_causal_conv(torch.zeros(8, 6).t(), w, off, y_out=g)
    with pytest.raises(TypeError, match="y_out"):
        pg.precog_conv_step(x, w, win, y_out=x.half())
    with pytest.raises(TypeError, match="windows"):
        pg.precog_conv_step(x, w, win.half(), y_out=g)
    with pytest.raises(ValueError, match="windows must be contiguous"):
        pg.precog_conv_step(x, w, torch.zeros(2, 1, 8, 3).transpose(2, 3), y_out=g)
    with pytest.raises(ValueError, match="weight"):
        pg.precog_conv_step(x, torch.zeros(9, 4), win, y_out=g)
    with pytest.raises(ValueError, match="out must be"):
        pg.precog_block_norm(x, out=x[:, :4])
    with pytest.raises(TypeError, match="out"):
        pg.precog_block_norm(x, out=x.half())
    with pytest.raises(TypeError, match="residual_out"):
        pg.precog_block_norm(x, residual=g, residual_out=g.bfloat16())
    with pytest.raises(ValueError, match="norm"):
        pg.precog_block_norm(x, out=x, norm="l2")
    with pytest.raises(ValueError, match="together"):
        pg.precog_adjust_logits(x, x, bias=g)
    with pytest.raises(ValueError, match="history_offsets"):
        pg.precog_adjust_logits(x, x, history=off)
    with pytest.raises(ValueError, match="need a history"):
        pg.precog_adjust_logits(x, x, repetition=g)
    with pytest.raises(ValueError, match="without mask"):
        pg.precog_adjust_logits(x, x, mask_rows=off)
    with pytest.raises(TypeError, match="out"):
        pg.precog_adjust_logits(x, x.half())
    with pytest.raises(ValueError, match="mask must be"):
        pg.precog_adjust_logits(x, g, mask=torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(TypeError, match="one dtype"):
        pg.scan_inputs(x, x.bfloat16(), torch.zeros(6, 16), torch.zeros(8, 16))
    with pytest.raises(TypeError, match="one dtype"):
        pg.scan_inputs(x, x, torch.zeros(6, 16), torch.zeros(8, 16), torch.zeros(6, 16).half())
    with pytest.raises(ValueError, match="GPU"):
        pg.scan_inputs(x, x, torch.zeros(6, 16), torch.zeros(8, 16))
    monkeypatch.setattr(pg, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="GPU"):
        pg.precog_causal_conv(x, w, off, y_out=g)
    with pytest.raises(ValueError, match="GPU"):
        pg.precog_block_norm(x, out=g)
    with pytest.raises(ValueError, match="GPU"):
        pg.precog_adjust_logits(x, g)


def test_packed_arguments_are_the_structures_bytes(lib):
    """The binding packs its arguments instead of filling a Structure: the same bytes, field by field."""
    import paper_2608_02560_gb300 as pg
    for cls in (pg.ConvArgs, pg.ScanStepArgs, pg.BlockNormArgs, pg.AdjustArgs):
        values = [1.5 if kind is ctypes.c_float else i + 3 for i, (_, kind) in enumerate(cls._fields_)]
        assert bytes(cls(*values)) == pg._packer(cls).pack(*values)
