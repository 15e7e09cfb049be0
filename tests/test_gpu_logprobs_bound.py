"""The bound that the warps of a row share while they raise it: rows in which every warp has entries for
the list until the very end, heads and tails of less than a vector among them. Indices are exact."""
import numpy as np
import pytest

import oracle
from tests._util import to_np
from tests.test_gpu_logprobs import _compare, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("R,V,k", [(3, 60013, 32), (700, 20007, 20), (1300, 9003, 32)])
def test_rows_that_rise_to_their_end(cuda_device, dtype, R, V, k):
    import torch
    dt = getattr(torch, dtype)
    gen = torch.Generator(device=cuda_device).manual_seed(R)
    x = torch.empty((R, V + 3), device=cuda_device)
    x[:] = torch.arange(V + 3, device=cuda_device) * (40.0 / V)       # steps of the 16-bit types: many ties
    x[1::3] = x[1::3].flip(1)
    x[2::3] += 3 * torch.rand((x[2::3].shape[0], V + 3), device=cuda_device, generator=gen)
    x = x.to(dt)[:, 1:V + 1]                                          # (rows begin and end within a vector)
    tokens = torch.randint(0, V, (R,), device=cuda_device, generator=gen)
    got = _run(cuda_device, x, tokens, 1.0, k)
    rows = [0, 1, 2, R // 2, R - 1]
    ref = oracle.token_logprobs(to_np(x[rows]), tokens[rows].tolist(), 1.0, k)
    _compare([g[rows] for g in got], ref, k)
    for _ in range(5):
        again = _run(cuda_device, x, tokens, 1.0, k)
        assert all(torch.equal(a, b) for a, b in zip(again, got))
    assert np.all(to_np(got[3]) <= 0)
