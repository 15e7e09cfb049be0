"""Log probabilities of given tokens, entropy and best entries against the fp64 definition.

Tolerances: the sums run over at most 2^17 terms in fp32, joined pairwise over the threads, so
their relative error stays below 2^-15 * 2^-6 = 5e-7, and a difference of logits up to 100 is off
by at most 100 * 2^-23: 3e-5 absolute covers log probabilities and entropies at the sizes here.
Indices are exact."""
import numpy as np
import pytest

import oracle
from tests._util import to_np

pytestmark = pytest.mark.gpu

TOL = 3e-5


def _run(dev, x, tokens, temperature=1.0, k=0, entropy=True):
    import torch
    import paper_2608_02560_gb300 as pg
    R = x.shape[0]
    lp = torch.full((R,), 9.0, device=dev)
    H = torch.full((R,), 9.0, device=dev) if entropy else None
    idx = torch.full((R, k), -9, dtype=torch.int64, device=dev) if k else None
    best = torch.full((R, k), 9.0, device=dev) if k else None
    pg.precog_token_logprobs(x, tokens, lp, entropy=H, top_idx=idx, top_logprob=best, temperature=temperature)
    return lp, H, idx, best


def _compare(got, ref, k):
    lp, H, idx, best = got
    for g, r in ((lp, ref[0]), (H, ref[1])) + (((best, ref[3]),) if k else ()):
        g = to_np(g)
        assert np.array_equal(np.isnan(g), np.isnan(r))
        assert np.array_equal(np.isinf(g), np.isinf(r))
        fine = np.isfinite(r)
        assert np.all(np.abs(g[fine] - r[fine]) <= TOL), float(np.max(np.abs(g[fine] - r[fine])))
    if k:
        assert np.array_equal(idx.cpu().numpy(), ref[2])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("R,V,pad,k,temp", [
    (1, 1, 0, 1, 1.0), (3, 7, 0, 7, 0.5), (2, 33, 3, 32, 1.0), (5, 1000, 1, 0, 1.0), (4, 32000, 0, 5, 1.0),
    (70, 5003, 5, 20, 1.7), (1, 131073, 0, 32, 1.0), (300, 257, 0, 1, 1.0), (2, 8191, 2, 9, 0.3)])
def test_matches_the_definition(cuda_device, dtype, R, V, pad, k, temp):
    import torch
    gen = torch.Generator(device=cuda_device).manual_seed(V + k)
    x = (3 * torch.randn((R, V + pad), device=cuda_device, generator=gen)).to(getattr(torch, dtype))
    x[:, V:] = float("nan")                       # the padding of the rows is nobody's
    x = x[:, :V]
    tokens = torch.randint(0, V, (R,), device=cuda_device, generator=gen)
    tokens[0] = V - 1
    ref = oracle.token_logprobs(to_np(x), tokens.tolist(), temp, k)
    _compare(_run(cuda_device, x, tokens, temp, k), ref, k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [9, 4097])
def test_masked_extreme_and_broken_rows(cuda_device, dtype, V):
    """-infinity, the type's lowest value, +infinity, NaN; all entries equal; one entry left."""
    import torch
    dt = getattr(torch, dtype)
    lowest = torch.finfo(dt).min
    x = torch.randn((10, V), device=cuda_device).to(dt)
    x[0] = float("-inf")
    x[1] = lowest
    x[2] = lowest
    x[2, V // 2] = 4.0
    x[3] = float("-inf")
    x[3, V - 1] = -2.0
    x[4, 3] = float("nan")
    x[5, 3] = float("inf")
    x[6] = 1.5
    x[7, ::2] = float("-inf")
    x[8] = torch.finfo(dt).max
    x[9] = 0.0
    x[9, 1::2] = -0.0
    tokens = torch.tensor([0, 1, V // 2, 0, 2, 3, 5, 1, 7, 4], device=cuda_device)
    ref = oracle.token_logprobs(to_np(x), tokens.tolist(), 1.0, 6)
    _compare(_run(cuda_device, x, tokens, 1.0, 6), ref, 6)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("R,V,k,temp", [(1300, 1001, 5, 1.0), (1217, 2100, 32, 0.7), (1250, 1, 1, 1.0), (700, 1001, 7, 1.0),
                                        (650, 2309, 0, 1.3), (1300, 515, 0, 1.0)])
def test_many_rows(cuda_device, dtype, R, V, k, temp):
    """As many rows as give each few warps, masked, extreme and broken ones among them."""
    import torch
    gen = torch.Generator(device=cuda_device).manual_seed(R + V + k)
    dt = getattr(torch, dtype)
    x = (3 * torch.randn((R, V), device=cuda_device, generator=gen)).to(dt)
    x[1::11] = float("-inf")
    x[2::11] = torch.finfo(dt).min
    x[3::11, V // 2] = float("nan")
    x[4::11, V // 3] = float("inf")
    x[5::11, ::2] = float("-inf")
    x[6::11] = 1.5
    x[7::11, 1:] = torch.finfo(dt).min
    x[8::11, :V - 1] = float("-inf")
    x[9::11] = torch.arange(V, device=cuda_device).to(dt) * 2.0 ** -6      # every entry enters the list
    tokens = torch.randint(-1, V, (R,), device=cuda_device, generator=gen)
    ref = list(oracle.token_logprobs(to_np(x), tokens.tolist(), temp, k))
    got = [g if g is None else to_np(g) for g in _run(cuda_device, x, tokens, temp, k)]
    # A difference d of logits is off by d * 2^-23: TOL is that up to 100. The log probabilities of
    # the seventh kind's masked entries lie far below, and beyond fp32's range are its -infinity.
    for i in (0, 3) if k else (0,):
        far = np.isfinite(ref[i]) & (ref[i] < -100)
        assert set(np.argwhere(far)[:, 0] % 11) <= {7}
        with np.errstate(over="ignore", invalid="ignore"):
            near = np.abs(got[i][far] - ref[i][far]) <= np.abs(ref[i][far]) * 2.0 ** -23
            assert np.all(near | (got[i][far] == ref[i][far].astype(np.float32)))
        got[i][far] = ref[i][far] = 0.0
    _compare([g if g is None else torch.from_numpy(g) for g in got], ref, k)


def test_sorted_rows_and_ties(cuda_device):
    """Rows in which every entry enters the list of the best, and rows of many equal entries."""
    import torch
    V = 20000
    x = torch.empty((4, V), device=cuda_device)
    x[0] = torch.arange(V, device=cuda_device) * 1e-3
    x[1] = -x[0]
    x[2] = (torch.arange(V, device=cuda_device) % 7).float()
    x[3] = (torch.arange(V, device=cuda_device) // 100 % 3).float()
    x = x.to(torch.bfloat16)
    tokens = torch.tensor([V - 1, 0, 6, 1], device=cuda_device)
    ref = oracle.token_logprobs(to_np(x), tokens.tolist(), 1.0, 32)
    _compare(_run(cuda_device, x, tokens, 1.0, 32), ref, 32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("temp", [1e-3, 30.0, 1e5, 1e36])
def test_temperatures(cuda_device, dtype, temp):
    """Rows with masked entries from nearly greedy to nearly uniform. Log probabilities scale with
    1 / temperature, and with them the rounding of the logits' differences."""
    import torch
    gen = torch.Generator(device=cuda_device).manual_seed(17)
    x = (2 * torch.randn((3, 3000), device=cuda_device, generator=gen)).to(getattr(torch, dtype))
    x[:, ::3] = float("-inf")
    x[1, 5] = torch.finfo(x.dtype).min
    x[2, 7] = torch.finfo(x.dtype).min / 2
    tokens = torch.tensor([1, 5, 7], device=cuda_device)
    lp, H, idx, best = _run(cuda_device, x, tokens, temp, 8)
    ref = oracle.token_logprobs(to_np(x), tokens.tolist(), temp, 8)
    assert np.array_equal(idx.cpu().numpy(), ref[2])
    for g, r in ((lp, ref[0]), (H, ref[1]), (best, ref[3])):
        g = to_np(g)
        r32 = np.where(np.abs(r) > 3.5e38, -np.inf, r)            # beyond fp32
        assert np.array_equal(np.isinf(g), np.isinf(r32))
        fine = np.isfinite(r32)
        assert np.all(np.abs(g[fine] - r32[fine]) <= TOL + 4 * 2.0 ** -24 * np.abs(r32[fine]) * max(1.0, 20 / temp))


def test_tokens_that_are_none_or_outside(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    x = torch.randn((4, 50), device=cuda_device)
    lp, H, _, _ = _run(cuda_device, x, torch.tensor([-1, 50, -2, 3], device=cuda_device))
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    assert float(lp[0]) == 0.0 and bool(torch.isnan(lp[1:3]).all()) and bool(torch.isfinite(H).all())
    ref = oracle.token_logprobs(to_np(x[3:]), [3])
    assert abs(float(lp[3]) - ref[0][0]) < TOL
    lp2, none, _, _ = _run(cuda_device, x, torch.tensor([-1, 1, 2, 3], device=cuda_device), entropy=False)
    assert none is None and float(lp2[3]) == float(lp[3]) and pg.precog_device_status()[0] == 0


def test_rows_past_32_bits(cuda_device):
    import torch
    V, R = 2 ** 20 + 1, 2100
    x = torch.empty((R, V), dtype=torch.bfloat16, device=cuda_device)
    x[-1].normal_()
    row = x[-1:].clone()
    x[:-1] = 0
    tokens = torch.full((R,), 12345, dtype=torch.int64, device=cuda_device)
    big = _run(cuda_device, x, tokens, 1.0, 3)
    one = _run(cuda_device, row, tokens[:1], 1.0, 3)
    ref = oracle.token_logprobs(to_np(row), [12345], 1.0, 3)
    for a, b in zip(big, one):
        assert np.allclose(to_np(a[-1:]), to_np(b), rtol=0, atol=TOL)
    assert np.array_equal(big[2][-1:].cpu().numpy(), ref[2]) and abs(float(big[0][-1]) - ref[0][0]) < TOL
    assert abs(float(big[0][0]) + np.log(V)) < TOL
