"""Logits or temperatures for which the scaled maximum is far beyond what 24 bits resolve.

Tolerance: as in test_gpu_logprobs_offsets.py."""
import pytest

from tests.test_gpu_logprobs_offsets import _exactly

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,top,temp", [
    ("float32", 1e8, 1.0), ("float32", 3e9, 1.0), ("float32", -3e9, 1.0), ("float32", 1e12, 1.0), ("float32", -1e20, 1.0),
    ("float32", 1e30, 1e12), ("float32", 700.0, 1e-7), ("bfloat16", 1e10, 1.0), ("bfloat16", -1e10, 1.0),
    ("bfloat16", 90.0, 1e-8), ("float16", 6e4, 1e-5), ("float16", -6e4, 1e-5), ("float32", 1e6, 1e6), ("float32", 5.0, 1e30)])
@pytest.mark.parametrize("R,V,k", [(5, 9001, 8), (700, 1001, 3), (1300, 515, 5)])
def test_large_scaled_maxima(cuda_device, dtype, top, temp, R, V, k):
    """A few entries at or one step below the row's largest, the others far below; rows of one value."""
    import torch
    dt = getattr(torch, dtype)
    gen = torch.Generator(device=cuda_device).manual_seed(R)
    first = torch.tensor(top, dtype=dt)
    below = torch.nextafter(first.float(), torch.tensor(float("-inf"))).to(dt) if dt == torch.float32 else first
    x = torch.full((R, V), float(first) - 3 * abs(float(first)) if dt != torch.float16 else -6.5e4, device=cuda_device).to(dt)
    at = torch.randint(0, V, (R, 7), device=cuda_device, generator=gen)
    x.scatter_(1, at, float(below))
    x.scatter_(1, at[:, :3], float(first))
    x[1] = float(first)
    tokens = at[:, 0].contiguous()
    _exactly(x, tokens, temp, k, cuda_device)
