"""Calls on a stream that is not torch's current one, whose workspace the binding allocates: nothing that
is allocated meanwhile meets it."""
import pytest

from tests.test_gpu_delta import TOL_PAIR, _ref, _tensors
from tests._util import rel_err, to_np

pytestmark = pytest.mark.gpu


def _busy(side):
    """A few milliseconds of copies, so that what follows on the stream has not begun yet."""
    import torch
    with torch.cuda.stream(side):
        a, b = (torch.empty(2 ** 28, dtype=torch.uint8, device="cuda") for _ in range(2))
        for _ in range(20):
            b.copy_(a)


def test_a_cut_scan_on_a_side_stream(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    T = 6000
    q, k, v, g, beta, off = _tensors([T], 1, 2, 64, 64, torch.bfloat16, cuda_device, 61, rate=0.02)
    inputs = pg.delta_inputs(q, k, v, g, beta)
    need = pg.precog_delta_scan_workspace_size(inputs, 1, T)
    assert need > 0
    s, y = torch.empty((1, 1, 2, 64, 64), device=cuda_device), torch.empty((T, 2, 64), device=cuda_device)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy(side)
    pg.precog_delta_scan(inputs, off, T, states_out=s, y_out=y, stream=side)
    others = [torch.full((need // 4,), float("nan"), device=cuda_device) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(bool(torch.isnan(o).all()) for o in others)
    ref_S, ref_y = _ref(q, k, v, g, beta, off)
    assert rel_err(to_np(s[:, 0]), ref_S) < TOL_PAIR and rel_err(to_np(y), ref_y) < TOL_PAIR
    assert pg.precog_device_status()[0] == 0


def test_retrieval_on_a_side_stream(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    M, Q, dim = 20011, 5, 64
    index, queries = (torch.randn((n, dim), device=cuda_device) for n in (M, Q))
    want, want_k = torch.empty(Q, dtype=torch.int64, device=cuda_device), torch.empty((Q, 3), dtype=torch.int64, device=cuda_device)
    pg.precog_retrieve(index, queries, want)
    pg.precog_retrieve_topk(index, queries, 3, want_k)
    sizes = {pg.precog_retrieve_workspace_size(M, dim, Q), pg.precog_retrieve_topk_workspace_size(M, dim, Q)}
    got, got_k = torch.full_like(want, -7), torch.full_like(want_k, -7)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy(side)
    pg.precog_retrieve(index, queries, got, stream=side)
    pg.precog_retrieve_topk(index, queries, 3, got_k, stream=side)
    others = [torch.full((n,), 255, dtype=torch.uint8, device=cuda_device) for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    assert all(bool((o == 255).all()) for o in others)
    assert torch.equal(got, want) and torch.equal(got_k, want_k)
