"""Logits with a large common part, and small temperatures: what counts is their differences.

Tolerance: differences of such logits are exact or rounded once, a log probability is the sum of two
numbers with four roundings each, of 2^-24 of their size, and the sums' logarithm is within 2^-23 of
its 17 and of the exponentials' 2^-22: 2^-22 |log p| + 1e-5. An entropy is a difference of two numbers
up to 17: 1e-5."""
import numpy as np
import pytest

import oracle
from tests._util import to_np
from tests.test_gpu_logprobs import _run

pytestmark = pytest.mark.gpu


def _exactly(x, tokens, temp, k, dev):
    ref = oracle.token_logprobs(to_np(x), tokens.tolist(), float(np.float32(temp)), k)
    lp, H, idx, best = _run(dev, x, tokens, temp, k)
    for got, r, rel in ((lp, ref[0], 2.0 ** -22), (H, ref[1], 0.0)) + (((best, ref[3], 2.0 ** -22),) if k else ()):
        got = to_np(got)
        assert np.array_equal(np.isfinite(got), np.isfinite(r))
        fine = np.isfinite(r)
        worst = np.abs(got[fine] - r[fine]) - rel * np.abs(r[fine])
        assert np.max(worst) <= 1e-5, float(np.max(worst))
    if k:
        assert np.array_equal(idx.cpu().numpy(), ref[2])


@pytest.mark.parametrize("R,V,k", [(3, 50257, 5), (700, 3001, 4), (1300, 2005, 6), (2, 90, 0)])
@pytest.mark.parametrize("offset", [-1e4, -30.0, 100.0, 1e3, 1e4])
def test_a_common_offset_changes_nothing(cuda_device, offset, R, V, k):
    import torch
    gen = torch.Generator(device=cuda_device).manual_seed(R)
    x = 2.5 * torch.randn((R, V), device=cuda_device, generator=gen) + offset
    tokens = torch.randint(0, V, (R,), device=cuda_device, generator=gen)
    _exactly(x, tokens, 1.0, k, cuda_device)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("temp", [1e-3, 0.05, 3.0])
def test_small_temperatures_lose_nothing(cuda_device, dtype, temp):
    import torch
    gen = torch.Generator(device=cuda_device).manual_seed(23)
    x = (40 + 3 * torch.randn((5, 9001), device=cuda_device, generator=gen)).to(getattr(torch, dtype))
    x[2, ::3] = float("-inf")
    x[3] += 200
    tokens = torch.tensor([1, 5, 7, 9000, 0], device=cuda_device)
    _exactly(x, tokens, temp, 8, cuda_device)
