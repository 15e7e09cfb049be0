"""Penalties, biases and masks on logits against the definition in 64 bits.

Bound: a quotient or product, a product and two differences, a sum: five roundings to fp32 of the magnitudes that
meet, then the output's own. Places of -infinity are exact."""
import numpy as np
import pytest

import oracle
from tests._layer import U, close
from tests._util import to_np

pytestmark = pytest.mark.gpu


def _words(bits):
    """bool [m, V] as int32 words."""
    import torch
    m, V = bits.shape
    b = np.zeros((m, (V + 31) // 32 * 32), dtype=np.uint64)
    b[:, :V] = bits
    w = (b.reshape(m, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32))


def _lists(lists, dev, dtype=None):
    import torch
    off = torch.tensor([0] + list(np.cumsum([len(v) for v in lists])), dtype=torch.int64, device=dev)
    flat = [i for v in lists for i in v]
    return torch.tensor(flat, dtype=dtype or torch.int64, device=dev), off


def _case(dev, R, V, dtype, seed, longest=60, rep=True, freq=True, pres=True, bias=5, masks=3, counts=True, pad=0):
    import torch
    r = np.random.default_rng(seed)
    x = torch.from_numpy(3.0 * r.standard_normal((R, V + pad)).astype(np.float32)).to(dev).to(getattr(torch, dtype))[:, pad:]
    history = [list(r.integers(-1, max(1, min(V, 9 if i % 2 else V)), r.integers(0, longest + 1))) for i in range(R)]
    c = dict(x=x, history=history, rep=r.uniform(0.7, 1.9, R) if rep else None, freq=r.uniform(-0.5, 0.9, R) if freq else None,
             pres=r.uniform(-0.5, 0.9, R) if pres else None, start=r.integers(-3, longest, R) if counts else None, biases=None,
             bits=None, rows=None)
    if bias:
        c["biases"] = [[(int(i), float(np.float32(b))) for i, b in zip(r.integers(-1, V, r.integers(0, bias + 1)),
                                                                       r.standard_normal(bias))] for _ in range(R)]
    if masks:
        c["bits"] = r.random((masks, V)) < 0.5
        c["bits"][0] = False                                    # nothing is allowed
        c["rows"] = r.integers(-1, masks, R)
    for k in ("rep", "freq", "pres"):
        if c[k] is not None:
            c[k] = c[k].astype(np.float32)
    return c


def _run(dev, c, out=None):
    import torch
    import paper_2608_02560_gb300 as pg
    dv = lambda a, t: None if a is None else torch.from_numpy(np.asarray(a).astype(t)).to(dev)  # noqa: E731
    h, off = _lists(c["history"], dev)
    bi = bv = bo = None
    if c["biases"] is not None:
        bi, bo = _lists([[i for i, _ in v] for v in c["biases"]], dev)
        bv, _ = _lists([[b for _, b in v] for v in c["biases"]], dev, torch.float32)
    out = torch.empty(c["x"].shape, dtype=c["x"].dtype, device=dev) if out is None else out
    pg.precog_adjust_logits(c["x"], out, history=h, history_offsets=off, count_from=dv(c["start"], np.int64),
                            repetition=dv(c["rep"], np.float32), frequency=dv(c["freq"], np.float32),
                            presence=dv(c["pres"], np.float32), bias_idx=bi, bias=bv, bias_offsets=bo,
                            mask=None if c["bits"] is None else _words(c["bits"]).to(dev), mask_rows=dv(c["rows"], np.int64))
    return out


def _check(c, out, x):
    R, V = x.shape
    allowed = None
    if c["bits"] is not None:
        rows = np.arange(R) if c["rows"] is None else c["rows"]
        allowed = [None if m < 0 else set(np.flatnonzero(c["bits"][m])) for m in rows]
    ref = oracle.adjust_logits(x, c["history"], c["start"], c["rep"], c["freq"], c["pres"], c["biases"], allowed)
    size = max([1.0] + [float(np.abs(c[k]).max()) for k in ("freq", "pres") if c[k] is not None])
    times = np.array([[h.count(i) for i in range(V)] if V < 2000 else [len(h)] * V for h in c["history"]])
    most = max([0.0] + [abs(b) for v in c["biases"] or [] for _, b in v])
    with np.errstate(invalid="ignore"):
        bound = 5 * U * (2 * np.where(np.isfinite(x), np.abs(x), 0) + size * (times + 1) + most)
    close(to_np(out), ref, bound, out.dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("R,V,pad", [(1, 1, 0), (3, 31, 0), (5, 32, 3), (7, 33, 1), (64, 257, 5), (2, 8191, 8), (3, 8193, 0),
                                     (3, 16400, 7)])
def test_rows_match_the_definition(cuda_device, dtype, R, V, pad):
    import paper_2608_02560_gb300 as pg
    c = _case(cuda_device, R, V, dtype, 5 * R + V, pad=pad)
    out = _run(cuda_device, c)
    assert pg.precog_device_status()[0] == 0
    _check(c, out, to_np(c["x"]))
    # in place: the same bits, and nothing beside the rows
    import torch
    x = c["x"]
    again = dict(c, x=x.clone() if not pad else torch.cat([torch.full_like(x[:, :pad], 5.0), x], 1)[:, pad:])
    _run(cuda_device, again, out=again["x"])
    assert torch.equal(again["x"], out)
    if pad:
        assert bool((again["x"].as_strided((R, pad), (V + pad, 1), 0) == 5.0).all())


@pytest.mark.parametrize("V", [2048, 2049, 6000])
def test_few_rows_with_long_lists(cuda_device, V):
    c = _case(cuda_device, 4, V, "float32", V)
    r = np.random.default_rng(V)
    c["history"][1] = list(r.integers(0, V, 20_000))
    c["biases"][2] = [(int(i), float(np.float32(b))) for i, b in zip(r.integers(0, V, 5000), r.standard_normal(5000))]
    _check(c, _run(cuda_device, c), to_np(c["x"]))


@pytest.mark.parametrize("on", ["rep", "freq", "pres", "bias", "masks", "nothing"])
def test_each_alone(cuda_device, on):
    c = _case(cuda_device, 6, 500, "float32", 3, rep=on == "rep", freq=on == "freq", pres=on == "pres",
              bias=7 if on == "bias" else 0, masks=4 if on == "masks" else 0, counts=False)
    _check(c, _run(cuda_device, c), to_np(c["x"]))


def test_long_histories_count_exactly(cuda_device):
    """5000 times one token, counted from 1000 on, in one row among short ones."""
    c = _case(cuda_device, 4, 300, "float32", 9, bias=0, masks=0)
    c["history"][2], c["start"][2] = [7] * 5000 + [299, -1, 0], 1000
    _check(c, _run(cuda_device, c), to_np(c["x"]))


def test_masks_of_rows_themselves_and_the_answers_distribution(cuda_device):
    """Without mask_rows row r has mask r; a row whose mask leaves nothing has no distribution; infinities and NaN in
    masked places are gone."""
    import torch
    import paper_2608_02560_gb300 as pg
    c = _case(cuda_device, 3, 100, "float32", 4, masks=3, bias=0)
    c["rows"] = None
    banned = np.flatnonzero(~c["bits"][1])
    c["x"][1, int(banned[0])], c["x"][1, int(banned[1])], c["x"][0, 5] = float("nan"), float("inf"), float("nan")
    out = _run(cuda_device, c)
    _check(c, out, to_np(c["x"]))
    lp, H = torch.empty(3, device=cuda_device), torch.empty(3, device=cuda_device)
    tok = torch.tensor([0, int(np.flatnonzero(c["bits"][1])[0]), int(np.flatnonzero(c["bits"][2])[0])], device=cuda_device)
    pg.precog_token_logprobs(out, tok, lp, H)
    assert bool(torch.isnan(lp[0])) and bool(torch.isfinite(lp[1:]).all()) and bool(torch.isfinite(H[1:]).all())


def test_values_that_are_not_finite_stay_in_their_places(cuda_device):
    c = _case(cuda_device, 3, 64, "bfloat16", 6, masks=0, bias=0)
    c["x"][0, 3], c["x"][1, 4], c["x"][2, 5] = float("nan"), float("inf"), float("-inf")
    for r, i in ((0, 3), (1, 4), (2, 5)):
        c["history"][r] += [i, i]
    _check(c, _run(cuda_device, c), to_np(c["x"]))


def test_bad_tokens_lists_and_masks_are_ignored_and_flagged(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    d = cuda_device
    x = torch.randn((3, 50), device=d)
    rep = torch.full((3,), 2.0, device=d)
    i64 = lambda *v: torch.tensor(v, dtype=torch.int64, device=d)  # noqa: E731
    out = torch.empty_like(x)
    plain = lambda **kw: pg.precog_adjust_logits(x, out, **kw)  # noqa: E731
    plain(history=i64(50, -2, 1 << 40, 3), history_offsets=i64(0, 0, 4, 4), repetition=rep)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    want = x.clone()
    want[1, 3] = x[1, 3] / 2 if x[1, 3] > 0 else x[1, 3] * 2
    assert torch.equal(out, want)
    for off in (i64(0, 3, 2, 4), i64(-1, 0, 0, 0), i64(0, 0, 0, 5), i64(0, 1 << 62, -(1 << 62), 0)):
        plain(history=i64(1, 1, 1, 1), history_offsets=off, repetition=rep)
        assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_OFFSETS)
        plain(bias_idx=i64(1, 1, 1, 1), bias=rep.new_ones(4), bias_offsets=off)
        assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_OFFSETS)
    plain(bias_idx=i64(50, -1), bias=rep.new_ones(2), bias_offsets=i64(0, 2, 2, 2))
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX) and torch.equal(out, x)
    plain(mask=torch.zeros((2, 2), dtype=torch.int32, device=d), mask_rows=i64(2, -2, 1))
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    assert torch.equal(out[:2], x[:2]) and bool((out[2] == float("-inf")).all())
    # no masks, no list entries at all
    empty = torch.empty(0, dtype=torch.int64, device=d)
    plain(mask=torch.zeros((0, 2), dtype=torch.int32, device=d), mask_rows=i64(-1, -1, -1), history=empty,
          history_offsets=i64(0, 0, 0, 0), repetition=rep, bias_idx=empty, bias=rep.new_ones(0), bias_offsets=i64(0, 0, 0, 0))
    assert pg.precog_device_status()[0] == 0 and torch.equal(out, x)


@pytest.mark.parametrize("dtype,V,pad", [("bfloat16", 30_011, 5), ("float32", 30_020, 0), ("float16", 30_008, 8), ("bfloat16", 131_075, 1)])
def test_a_batch_of_many_logits(cuda_device, dtype, V, pad):
    """More than 152 * 2 * 16,384 logits go through a copy and a launch behind it. Rows among them whose tokens do not fit
    in its table (20,000 different ones), with one token 30,000 times, and with 9000 biases, some of them twice."""
    import torch
    import paper_2608_02560_gb300 as pg
    R = 170 if V < 100_000 else 45
    c = _case(cuda_device, R, V, dtype, V + pad, longest=200, pad=pad)
    r = np.random.default_rng(3)
    c["history"][3] = list(r.permutation(V)[:20_000])
    c["history"][7] = [V - 1] * 30_000 + [0, -1]
    c["history"][11] = list(r.integers(0, V, 9000))
    c["start"][[3, 7, 11]] = 5000
    c["biases"][5] = [(int(i), float(np.float32(b))) for i, b in zip(r.integers(0, V, 9000), r.standard_normal(9000))]
    c["biases"][3] = c["biases"][5][:500]
    out = _run(cuda_device, c)
    assert pg.precog_device_status()[0] == 0
    _check(c, out, to_np(c["x"]))
    again = dict(c, x=c["x"].clone())
    _run(cuda_device, again, out=again["x"])
    assert torch.equal(again["x"], out)


@pytest.mark.parametrize("dtype,pad", [("bfloat16", 0), ("bfloat16", 3), ("float32", 2), ("float16", 8)])
def test_masks_alone_on_many_logits(cuda_device, dtype, pad):
    import paper_2608_02560_gb300 as pg
    c = _case(cuda_device, 45, 131_075, dtype, 2, longest=0, rep=False, freq=False, pres=False, bias=0, counts=False, pad=pad)
    out = _run(cuda_device, c)
    assert pg.precog_device_status()[0] == 0
    want = to_np(c["x"]).copy()
    for r, m in enumerate(c["rows"]):
        if m >= 0:
            want[r, ~c["bits"][m]] = -np.inf
    assert np.array_equal(to_np(out), want)


def test_pairs_of_launches_in_order_captured_and_at_once(cuda_device):
    """Many logits: call upon call without a wait between them, each on what the last one left; the same captured and
    replayed; and two streams at once. All give the bits of calls that are waited for."""
    import torch
    import paper_2608_02560_gb300 as pg
    d, R, V = cuda_device, 60, 30_011
    gen = torch.Generator(device=d).manual_seed(8)
    x = torch.randn((R, V), device=d, generator=gen).bfloat16()
    history = torch.randint(0, V, (R * 500,), device=d, generator=gen)
    args = dict(history=history, history_offsets=500 * torch.arange(R + 1, device=d), bias_idx=history[::50].contiguous(),
                bias=torch.randn(R * 10, device=d, generator=gen), bias_offsets=10 * torch.arange(R + 1, device=d),
                repetition=1 + torch.rand(R, device=d, generator=gen), frequency=torch.rand(R, device=d, generator=gen),
                presence=torch.rand(R, device=d, generator=gen))

    def chain(buf, wait):
        a, b, lp = buf
        for i in range(6):      # in place, over to the other buffer, back, and read out
            pg.precog_adjust_logits(a, a, **args)
            pg.precog_adjust_logits(a, b, **args)
            pg.precog_adjust_logits(b, a, **args)
            pg.precog_token_logprobs(a, history[:R], lp[i])
            if wait:
                torch.cuda.synchronize()

    buffers = lambda: (x.clone(), torch.zeros_like(x), torch.zeros((6, R), device=d))  # noqa: E731
    want, got = buffers(), buffers()
    chain(want, True)
    chain(got, False)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    captured, g = buffers(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        chain(captured, False)
    for _ in range(3):
        captured[0].copy_(x)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, captured))
    sides, streams = [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for side, stream in zip(sides, streams):
        with torch.cuda.stream(stream):
            chain(side, False)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for side in sides for p, q in zip(want, side))
    assert pg.precog_device_status()[0] == 0


def test_calls_of_one_input_repeat_bit_for_bit(cuda_device):
    import torch
    c = _case(cuda_device, 40, 9001, "bfloat16", 8, longest=3000)
    first = _run(cuda_device, c)
    assert all(torch.equal(first, _run(cuda_device, c)) for _ in range(3))


def test_rows_beyond_32_bits(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    d, R, V = cuda_device, 33_000, 131_075
    x = torch.zeros((R, V), dtype=torch.bfloat16, device=d)
    assert x.numel() > 1 << 32
    off = torch.zeros(R + 1, dtype=torch.int64, device=d)
    off[-1] = 2
    pg.precog_adjust_logits(x, x, history=torch.tensor([V - 1, 0], device=d), history_offsets=off,
                            presence=torch.ones(R, device=d))
    assert pg.precog_device_status()[0] == 0
    assert float(x[-1, 0]) == -1.0 and float(x[-1, -1]) == -1.0 and int(torch.count_nonzero(x)) == 2
