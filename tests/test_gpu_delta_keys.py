"""Keys that come back, small keys and the ends of beta's range, in chunks (whole sequences and cut ones).

Tolerances, max |gpu - ref| / max |ref|. An operand carried as two bf16 numbers is off by at most 2^-17
of itself, with no preferred sign.
* ORDINARY, unit keys that differ, betas below 1: five such products follow one another, each sum's terms
  of decreasing size: sqrt(5) 2^-17 = 1.7e-5, taken as 2e-5.
* TOL_PAIR (1.5e-4), any unit keys, betas in [0, 1]: no entry of the correction's inverse exceeds 1, the
  up to 64 terms of a token's correction may all be as large as it: sqrt(64) * 2^-17 = 6e-5 a chunk, of
  which the next corrections keep a part: twice that and a little.
* REFLECTED, betas up to 2: an entry of the inverse may be 4, and no chunk takes back what another left:
  64 * 4 * 2^-17 = 2e-3 a chunk if the roundings all agree, times the number of chunks."""
import numpy as np
import pytest

from tests._util import rel_err, to_np
from tests.test_gpu_delta import TOL_PAIR, _ref

pytestmark = pytest.mark.gpu

ORDINARY = 2e-5
REFLECTED = 2e-3


def _draw(kind, betas, decay, T, dk, dv, dev):
    import torch
    r = np.random.default_rng(1)

    def unit(x):
        return torch.tensor(x / np.linalg.norm(x, axis=-1, keepdims=True)).float().to(torch.bfloat16)
    q = unit(r.standard_normal((T, dk)))
    if kind == "different":
        k = unit(r.standard_normal((T, dk)))
    elif kind == "one":
        k = unit(r.standard_normal((1, dk))).expand(T, dk).contiguous()
    elif kind == "close":
        k = unit(r.standard_normal((1, dk)) + 0.3 * r.standard_normal((T, dk)))
    else:
        k = unit(r.standard_normal((4, dk)))[r.integers(0, 4, T)].contiguous()
    v = torch.tensor(r.standard_normal((T, dv))).to(torch.bfloat16)
    z = r.standard_normal(T)
    beta = np.full(T, float(betas)) if betas in ("1", "2") else float(betas[0]) / (1 + np.exp(-z))
    g = -decay * np.log1p(np.exp(r.standard_normal(T) - 2))
    S0 = torch.tensor(r.standard_normal((1, 1, 1, dv, dk))).float()
    f = lambda x: torch.tensor(x).float()[:, None].to(dev)  # noqa: E731
    return q[:, None].to(dev), k[:, None].to(dev), v[:, None].to(dev), f(g), f(beta), S0.to(dev)


def _errors(kind, betas, decay, T, dk, dev):
    import torch
    import paper_2608_02560_gb300 as pg
    dv = 128
    q, k, v, g, beta, S0 = _draw(kind, betas, decay, T, dk, dv, dev)
    off = torch.tensor([0, T], device=dev)
    s, alone = torch.empty_like(S0), torch.empty_like(S0)
    y = torch.empty((T, 1, dv), device=dev)
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, T, bank=S0, states_out=s, y_out=y)
    pg.precog_delta_scan(pg.delta_inputs(None, k, v, g, beta), off, T, bank=S0, states_out=alone)
    assert pg.precog_device_status()[0] == 0
    ref_S, ref_y = _ref(q, k, v, g, beta, off, to_np(S0[:, 0]))
    return [rel_err(to_np(a), b) for a, b in ((s[:, 0], ref_S), (alone[:, 0], ref_S), (y, ref_y))]


@pytest.mark.parametrize("decay", [0.0, 0.05])
@pytest.mark.parametrize("T,dk", [(256, 128), (1000, 64), (4096, 64)])
def test_keys_that_differ(cuda_device, T, dk, decay):
    assert max(_errors("different", "1 sigmoid", decay, T, dk, cuda_device)) < ORDINARY


@pytest.mark.parametrize("betas", ["1 sigmoid", "1"])
@pytest.mark.parametrize("kind", ["different", "one", "close", "four"])
@pytest.mark.parametrize("T,dk,decay", [(256, 128, 0.0), (1000, 128, 0.05), (1000, 8, 0.0), (1000, 64, 0.0), (4096, 64, 0.0),
                                        (4096, 128, 0.01)])
def test_any_keys_with_betas_up_to_one(cuda_device, T, dk, decay, kind, betas):
    assert max(_errors(kind, betas, decay, T, dk, cuda_device)) < TOL_PAIR


@pytest.mark.parametrize("betas", ["2 sigmoid", "2"])
@pytest.mark.parametrize("kind", ["different", "one", "close", "four"])
@pytest.mark.parametrize("T,dk,decay", [(256, 128, 0.0), (640, 64, 0.05), (640, 8, 0.0), (2048, 128, 0.01)])
def test_betas_up_to_two(cuda_device, T, dk, decay, kind, betas):
    assert max(_errors(kind, betas, decay, T, dk, cuda_device)) < REFLECTED * (T // 64)


def test_fp32_inputs_keep_more(cuda_device):
    """The same keys and betas in fp32, token by token."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, S0 = _draw("one", "2", 0.0, 1000, 64, 128, cuda_device)
    q, k, v = q.float(), k.float(), v.float()
    off, s = torch.tensor([0, 1000], device=cuda_device), torch.empty_like(S0)
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, 1000, bank=S0, states_out=s)
    ref_S, _ = _ref(q, k, v, g, beta, off, to_np(S0[:, 0]))
    assert rel_err(to_np(s[:, 0]), ref_S) < 1e-5
