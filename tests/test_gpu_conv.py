"""The causal convolution over ragged sequences and for single tokens, against the fp64 definition (bounds:
tests/_layer.py). Windows are copies and have to be equal bit for bit."""
import numpy as np
import pytest

import oracle
from tests._layer import close, conv_bound
from tests._util import to_np

pytestmark = pytest.mark.gpu


def _rn(dev, seed):
    import torch
    gen = torch.Generator(device=dev).manual_seed(seed)
    return lambda *s: torch.randn(s, device=dev, generator=gen)


def _offsets(lens, dev, first=0):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]) + first, dtype=torch.int64, device=dev)


def _reference(x, w, off, b, silu, before):
    args = to_np(x), to_np(w), off.cpu().numpy(), None if b is None else to_np(b), silu, before
    y, behind = oracle.causal_conv(*args)
    return y, behind, conv_bound(*args, y, x.dtype)


CASES = [
    # lens, dim, K, bias, silu, bank
    ([1], 8, 4, True, True, False),
    ([64], 2048, 4, True, True, True),
    ([5, 0, 1, 2, 3, 0, 33, 32, 31, 130], 72, 4, True, True, True),
    ([0, 7, 1, 2, 64, 65], 136, 3, False, True, True),
    ([3, 1, 0, 40], 1032, 2, True, False, True),
    ([200, 1, 513], 264, 4, False, False, False),
    ([0, 0, 0], 64, 4, True, True, True),
    ([1] * 300, 16, 4, True, True, True),
    ([2500, 3], 40, 4, True, True, True),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("lens,dim,K,bias,silu,bank", CASES)
def test_sequences_match_the_definition(cuda_device, dtype, lens, dim, K, bias, silu, bank):
    import torch
    import paper_2608_02560_gb300 as pg
    d, dt, n, L, layer = cuda_device, getattr(torch, dtype), len(lens), 3, 1
    rn = _rn(d, 7 + sum(lens) + dim)
    T = sum(lens)
    x, w = rn(T, dim).to(dt), rn(dim, K)
    b = rn(dim) if bias else None
    off = _offsets(lens, d)
    table = idx = before = None
    if bank:
        table = rn(n + 2, L, K - 1, dim).to(dt)
        idx = torch.tensor([(3 * c) % (n + 3) - 1 for c in range(n)], dtype=torch.int64, device=d)
        before = [to_np(table[i, layer]) if i >= 0 else np.zeros((K - 1, dim)) for i in idx.tolist()]
    out = torch.full((n, L, K - 1, dim), 7.0, dtype=dt, device=d)
    y = torch.full((T, dim), float("nan"), dtype=dt, device=d)
    pg.precog_causal_conv(x, w, off, bias=b, silu=silu, bank=table, idx=idx, layer=layer, windows_out=out, y_out=y)
    assert pg.precog_device_status()[0] == 0
    ref, behind, bound = _reference(x, w, off, b, silu, before)
    close(to_np(y), ref, bound, dt)
    assert np.array_equal(to_np(out[:, layer]), behind)
    assert bool((out[:, 0] == 7.0).all()) and bool((out[:, 2] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_strides_rows_outside_and_broken_neighbours(cuda_device, dtype):
    """x and y are slices of one buffer; rows before and behind the sequences hold NaN, whose y rows stay; a
    sequence that ends in NaN touches no other."""
    import torch
    import paper_2608_02560_gb300 as pg
    d, dt = cuda_device, getattr(torch, dtype)
    rn = _rn(d, 3)
    wide = rn(300, 3 * 80 + 16).to(dt)
    x, y = wide[:, 16:96], wide[:, 176:256]
    w, b = rn(80, 4), rn(80)
    off = _offsets([50, 3, 0, 1, 100], d, first=9)
    end = int(off[-1])
    x[:9], x[end:] = float("nan"), float("inf")
    x[58] = float("nan")                       # the first sequence's last token
    before = wide.clone()
    pg.precog_causal_conv(x, w, off, bias=b, y_out=y)
    assert pg.precog_device_status()[0] == 0
    ref, _, bound = _reference(x, w, off, b, True, None)
    assert np.isnan(ref[58]).all() and np.isfinite(ref[9:58]).all() and np.isfinite(ref[59:end]).all()
    close(to_np(y[9:end]), ref[9:end], bound[9:end], dt)
    assert torch.equal(y[:9], before[:9, 176:256]) and torch.equal(y[end:], before[end:, 176:256])
    for lo, hi in ((0, 176), (256, 256)):
        assert torch.equal(wide[:, lo:hi].nan_to_num(5.0), before[:, lo:hi].nan_to_num(5.0))


def test_bad_offsets_and_bank_rows_are_flagged(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    d = cuda_device
    rn = _rn(d, 4)
    x, w = rn(400, 64), rn(64, 4)
    y = torch.full((400, 64), 3.0, device=d)
    out = torch.full((3, 1, 3, 64), 7.0, device=d)
    # decreasing, and beyond T: skipped; the first sequence is whole
    off = torch.tensor([5, 90, 60, 401], dtype=torch.int64, device=d)
    pg.precog_causal_conv(x, w, off, windows_out=out, y_out=y)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_OFFSETS)
    ref, behind, bound = _reference(x, w, off[:2], None, True, None)
    close(to_np(y[5:90]), ref[5:90], bound[5:90], x.dtype)
    assert bool((y[:5] == 3.0).all()) and bool((y[90:] == 3.0).all()) and bool((out[1:] == 7.0).all())
    for bad in ([-1, 5, 9, 12], [0, 1 << 40, 9, 12], [-(1 << 62), 1 << 62, -5, 12], [400, 300, 200, 100]):
        pg.precog_causal_conv(x, w, torch.tensor(bad, dtype=torch.int64, device=d), windows_out=out, y_out=y)
        assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_OFFSETS)
    # rows outside the bank: zeros
    off = _offsets([40, 40, 40], d)
    bank = rn(2, 1, 3, 64)
    pg.precog_causal_conv(x, w, off, bank=bank, idx=torch.tensor([-2, 2, 1 << 50], dtype=torch.int64, device=d), y_out=y)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    ref, _, bound = _reference(x[:120], w, off, None, True, None)
    close(to_np(y[:120]), ref, bound, x.dtype)
    pg.precog_causal_conv(x, w, off, bank=rn(0, 1, 3, 64), idx=torch.full((3,), -1, dtype=torch.int64, device=d), y_out=y)
    assert pg.precog_device_status()[0] == 0
    close(to_np(y[:120]), ref, bound, x.dtype)


@pytest.mark.parametrize("dtype,K", [("bfloat16", 4), ("float32", 3), ("bfloat16", 2)])
def test_a_cut_sequence_and_single_tokens_give_the_same_bits(cuda_device, dtype, K):
    """One call; two calls with the window between them (the injected chunk's); and token by token."""
    import torch
    import paper_2608_02560_gb300 as pg
    d, dt, T, D = cuda_device, getattr(torch, dtype), 70, 200
    rn = _rn(d, 5)
    x, w, b = rn(T, D).to(dt), rn(D, K), rn(D)
    whole, last = torch.empty_like(x), torch.empty((1, 1, K - 1, D), dtype=dt, device=d)
    pg.precog_causal_conv(x, w, _offsets([T], d), bias=b, windows_out=last, y_out=whole)
    for cut in (0, 1, 2, 3, 33, 69, 70):
        y, win, behind = torch.empty_like(x), torch.empty_like(last), torch.empty_like(last)
        pg.precog_causal_conv(x[:cut], w, _offsets([cut], d), bias=b, windows_out=win, y_out=y[:cut])
        pg.precog_causal_conv(x[cut:], w, _offsets([T - cut], d), bias=b, bank=win, windows_out=behind, y_out=y[cut:])
        assert torch.equal(y, whole) and torch.equal(behind, last)
    win, y = torch.zeros_like(last), torch.empty_like(x)
    for t in range(T):
        pg.precog_conv_step(x[t:t + 1], w, win, bias=b, y_out=y[t:t + 1])
    assert torch.equal(y, whole) and torch.equal(win, last)


@pytest.mark.parametrize("dtype,K", [("bfloat16", 4), ("float32", 4), ("bfloat16", 3), ("float32", 2)])
def test_long_segments_give_the_bits_of_short_calls(cuda_device, dtype, K):
    """Enough tokens for the longest segments, against calls of 500 tokens that hand the window on."""
    import torch
    import paper_2608_02560_gb300 as pg
    d, dt, D, lens = cuda_device, getattr(torch, dtype), 1032, [39_001, 0, 63, 64, 65, 2500]
    rn = _rn(d, 12)
    T = sum(lens)
    x, w, b = rn(T, D).to(dt), rn(D, K), rn(D)
    first = rn(len(lens), 1, K - 1, D).to(dt)
    y, behind = torch.empty_like(x), torch.empty_like(first)
    pg.precog_causal_conv(x, w, _offsets(lens, d), bias=b, bank=first, windows_out=behind, y_out=y)
    at, got = 0, torch.empty_like(x)
    for c, n in enumerate(lens):
        win = first[c:c + 1].clone()
        for t in range(at, at + n, 500):
            m, out = min(500, at + n - t), torch.empty_like(win)
            pg.precog_causal_conv(x[t:t + m], w, _offsets([m], d), bias=b, bank=win, windows_out=out, y_out=got[t:t + m])
            win = out
        assert torch.equal(win[0], behind[c])
        at += n
    assert torch.equal(got, y) and pg.precog_device_status()[0] == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,dim,K,silu", [(1, 8, 4, True), (1, 2048, 4, True), (5, 264, 3, False), (67, 1032, 4, True),
                                          (300, 136, 2, True), (256, 4104, 4, True), (300, 2056, 3, True),
                                          (200, 6152, 2, False)])
def test_steps_match_the_definition(cuda_device, dtype, n, dim, K, silu):
    import torch
    import paper_2608_02560_gb300 as pg
    d, dt, L, layer = cuda_device, getattr(torch, dtype), 2, 1
    rn = _rn(d, n + dim)
    wide = rn(n, dim + 24).to(dt)
    x, w, b = wide[:, 8:8 + dim], rn(dim, K), rn(dim)
    table = rn(n + 9, L, K - 1, dim).to(dt)
    slots = torch.randperm(n + 9, device=d)[:n].contiguous()
    if n > 1:
        slots[n // 2] = -1
    before = table.clone()
    y = torch.full((n, dim), 9.0, dtype=dt, device=d)
    pg.precog_conv_step(x, w, table, slots=slots, bias=b, silu=silu, layer=layer, y_out=y)
    assert pg.precog_device_status()[0] == 0
    live = (slots >= 0).cpu().numpy()
    rows = slots.cpu().numpy()[live]
    win = to_np(before[:, layer])[rows]
    m = len(rows)
    ref, behind, bound = _reference(x[torch.from_numpy(live).to(d)], w, torch.arange(m + 1), b, silu, win)
    close(to_np(y)[live], ref, bound, dt)
    assert bool((to_np(y)[~live] == 0).all())
    expect = to_np(before)
    expect[rows, layer] = behind
    assert np.array_equal(to_np(table), expect)
    inplace = x.clone()
    table.copy_(before)
    pg.precog_conv_step(inplace, w, table, slots=slots, bias=b, silu=silu, layer=layer, y_out=inplace)
    assert torch.equal(inplace, y) and np.array_equal(to_np(table), expect)


def test_slots_outside_the_table_are_idle_and_flagged(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    rn = _rn(cuda_device, 6)
    x, w, table = rn(4, 64), rn(64, 4), rn(3, 1, 3, 64)
    before, y = table.clone(), torch.full((4, 64), 9.0, device=cuda_device)
    pg.precog_conv_step(x, w, table, slots=torch.tensor([3, -2, 1 << 40, 1], device=cuda_device), y_out=y)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    assert bool((y[:3] == 0).all()) and bool((y[3] != 9.0).all())
    assert torch.equal(table[[0, 2]], before[[0, 2]]) and torch.equal(table[1, 0, :2], before[1, 0, 1:])
    assert torch.equal(table[1, 0, 2], x[3])


def test_offsets_beyond_32_bits(cuda_device):
    """A table of more than 2^32 elements: the last slot's window, and the first's."""
    import torch
    import paper_2608_02560_gb300 as pg
    d, slots, L, D = cuda_device, 44_000, 4, 8192
    table = torch.zeros((slots, L, 3, D), dtype=torch.bfloat16, device=d)
    assert table.numel() > 1 << 32
    rn = _rn(d, 8)
    x, w = rn(2, D).bfloat16(), rn(D, 4)
    table[0, 3], table[-1, 3] = rn(3, D).bfloat16(), rn(3, D).bfloat16()
    win = to_np(table[[0, slots - 1], 3])[::-1]
    y = torch.empty_like(x)
    pg.precog_causal_conv(x, w, _offsets([1, 1], d), bank=table, layer=3, y_out=y,
                          idx=torch.tensor([slots - 1, 0], dtype=torch.int64, device=d))
    ref, behind, bound = _reference(x, w, torch.arange(3), None, True, win)
    close(to_np(y), ref, bound, x.dtype)
    pg.precog_conv_step(x, w, table, slots=torch.tensor([slots - 1, 0], dtype=torch.int64, device=d), layer=3, y_out=y)
    close(to_np(y), ref, bound, x.dtype)
    assert np.array_equal(to_np(table[[slots - 1, 0], 3]), behind)
    assert pg.precog_device_status()[0] == 0
