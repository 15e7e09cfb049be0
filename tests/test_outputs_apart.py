"""Outputs that lie on a call's weights, lists or masks are refused on the host (a kernel may read them after it
has written there); beside them, in the gaps between strided rows too, they are not."""
import ctypes

import pytest

FAKE = 0x10000000  # a 16-byte aligned address that the host never dereferences
X, Y, W, T1, T2, FAR = (FAKE + i * 0x1000000 for i in range(6))   # 16 MiB apart
REFUSED, ROWS, LAYERS = 1, 3, 2


@pytest.fixture(scope="module")
def pg():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    pg.load_library()
    return pg


def _last_error(pg):
    return pg.load_library().precog_last_error().decode()


def _conv(pg, n_seqs=ROWS, T=100, offsets=W, idx=None, out=T1, y_stride=64, **kw):
    a = dict(dtype=pg.PRECOG_BF16, dim=64, kernel=4, silu=1, x=X, y=Y, x_stride=64, y_stride=y_stride, weight=FAR, bias=FAR + 4096)
    return pg.load_library().precog_causal_conv(ctypes.byref(pg.ConvArgs(**dict(a, **kw))), offsets, n_seqs, T, T2, 9, idx, out, 0, 1, None)


def _conv_step(pg, slots=W, windows=T1, **kw):
    a = dict(dtype=pg.PRECOG_BF16, dim=64, kernel=4, silu=1, x=X, y=Y, x_stride=64, y_stride=64, weight=FAR, bias=FAR + 4096)
    return pg.load_library().precog_conv_step(ctypes.byref(pg.ConvArgs(**dict(a, **kw))), ROWS, windows, 5, slots, 0, 1, None)


def _scan_step(pg, **kw):
    s = pg.ScanInputs(LAYERS, 64, 16, pg.PRECOG_BF16, 0, 0, X, X + 0x10000, X + 0x20000, X + 0x30000, X + 0x40000, 192, 48)
    a = dict(states=T1, n_slots=5, d_slots=W, layer0=0, L_total=LAYERS, skip=FAR, y_out=Y, y_dtype=pg.PRECOG_F32)
    return pg.load_library().precog_scan_step(ctypes.byref(s), ctypes.byref(pg.ScanStepArgs(**dict(a, **kw))), ROWS, None)


def _adjust(pg, **kw):
    a = dict(dtype=pg.PRECOG_BF16, vocab=100, stride=100, out_stride=100, logits=X, out=Y, n_history=50, n_bias=9, n_masks=4)
    lists = ("d_history", "d_history_offsets", "d_count_from", "d_repetition", "d_frequency", "d_presence", "d_bias_idx",
             "d_bias", "d_bias_offsets", "d_mask", "d_mask_rows")
    a.update({name: W + 4096 * i for i, name in enumerate(lists)})
    return pg.load_library().precog_adjust_logits(ctypes.byref(pg.AdjustArgs(**dict(a, **kw))), ROWS, None)


Y_END = Y + 99 * 128 + 128       # behind the last of 100 rows of 64 bf16


@pytest.mark.parametrize("kw", [
    dict(weight=Y), dict(weight=Y_END - 16), dict(weight=Y - 1024 + 16), dict(bias=Y + 256), dict(offsets=Y + 8), dict(idx=Y_END - 8),
    dict(weight=T1 + 1152 - 16), dict(bias=T1), dict(offsets=T1 - 24), dict(idx=T1 + 1144)])
def test_convolutions_outputs(pg, kw):
    before = pg.precog_launch_count()
    assert _conv(pg, **kw) == REFUSED and "share" in _last_error(pg)
    assert pg.precog_launch_count() == before


@pytest.mark.parametrize("kw", [
    dict(weight=Y), dict(weight=Y - 1008), dict(bias=Y + 2 * 128 + 112), dict(slots=Y + 376), dict(slots=Y - 16),
    dict(weight=T1 + 1904), dict(bias=T1 - 240), dict(slots=T1 + 1912)])
def test_convolution_steps_outputs(pg, kw):
    before = pg.precog_launch_count()
    assert _conv_step(pg, **kw) == REFUSED and "share" in _last_error(pg)
    assert pg.precog_launch_count() == before


Y_STEP, STATES = LAYERS * ROWS * 64 * 4, 5 * LAYERS * 64 * 16 * 4


@pytest.mark.parametrize("kw", [
    dict(skip=Y), dict(skip=Y + Y_STEP - 16), dict(skip=Y - 496), dict(d_slots=Y - 16), dict(d_slots=Y + Y_STEP - 8),
    dict(skip=T1 + STATES - 16), dict(d_slots=T1 + STATES - 8), dict(d_slots=T1 - 16)])
def test_scan_steps_outputs(pg, kw):
    before = pg.precog_launch_count()
    assert _scan_step(pg, **kw) == REFUSED and "share" in _last_error(pg)
    assert pg.precog_launch_count() == before


@pytest.mark.parametrize("name,size", [
    ("d_history", 400), ("d_history_offsets", 32), ("d_count_from", 24), ("d_repetition", 12), ("d_frequency", 12),
    ("d_presence", 12), ("d_bias_idx", 72), ("d_bias", 36), ("d_bias_offsets", 32), ("d_mask", 64), ("d_mask_rows", 24)])
def test_adjusted_logits(pg, name, size):
    before = pg.precog_launch_count()
    for at in (Y, Y + 2 * 200 + 192, Y - size + 8):
        assert _adjust(pg, **{name: at}) == REFUSED and "share" in _last_error(pg), at
    # rows of 200 bytes, 16,000 apart
    for at in (Y + 16000, Y + 32000 + 192, Y + 16000 - size + 8):
        assert _adjust(pg, out_stride=8000, stride=8000, **{name: at}) == REFUSED and "share" in _last_error(pg), at
    # in place it is the logits that are written
    assert _adjust(pg, out=X, **{name: X + 8}) == REFUSED
    assert pg.precog_launch_count() == before


def test_gaps_between_rows_belong_to_nobody(pg, monkeypatch):
    """(n_rows is what launches: without a GPU a call that passes its checks ends in a CUDA error instead.)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("addresses that only a host without a GPU may pass on")
    passed = lambda status: status not in (0, REFUSED, 2)  # noqa: E731
    for name in ("d_history", "d_mask"):
        for at in (Y + 200, Y + 16000 - 400, Y + 16000 + 200, Y + 32000 + 200, Y - 400):
            assert passed(_adjust(pg, out_stride=8000, stride=8000, **{name: at})), (name, at)
    assert passed(_conv(pg, weight=Y_END)) and passed(_conv(pg, weight=Y - 1024))
    assert passed(_conv(pg, weight=Y + 128, y_stride=1024)) and passed(_conv(pg, offsets=T1 + 1152))
    assert passed(_conv_step(pg, slots=Y + 3 * 128)) and passed(_scan_step(pg, skip=Y + Y_STEP)) and passed(_scan_step(pg, skip=Y - 512))
