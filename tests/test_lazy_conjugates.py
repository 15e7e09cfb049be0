"""Complex tensors that torch conjugates or negates lazily have other values than their memory: the binding
refuses them (``t.conj()`` is contiguous, and its pointer is its source's)."""
import pytest

N = 16


@pytest.fixture(scope="module")
def pg():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg


def _lazy(i):
    import torch
    z = torch.randn(2, 1, 8, N, dtype=torch.complex64)
    return [z.conj(), z[:1].conj(), torch._neg_view(z), z.conj().transpose(0, 1).transpose(0, 1)][i]


@pytest.mark.parametrize("i", range(4))
def test_tables_and_state_buffers(pg, monkeypatch, i):
    import torch
    t = _lazy(i)
    assert t.is_contiguous() and t.data_ptr() != t.resolve_conj().resolve_neg().data_ptr()
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    x, A, n = torch.zeros(2, 8), torch.zeros(1, 8, N, dtype=torch.complex64), t.shape[0]
    hand = pg.ScanInputs(1, 8, N, pg.PRECOG_F32, pg.PRECOG_A_COMPLEX, 0, 16, 16, 16, 16, 16, 16, 32)
    hand.rows, hand.device, hand._keepalive = n, -1, (x,)
    for take in (lambda: pg._dtype_code(t), lambda: pg.precog_scan_step(hand, t, y_out=torch.zeros(1, n, 8)),
                 lambda: pg.scan_inputs(x, x, torch.zeros(2, N), t[0], torch.zeros(2, N), a_kind=pg.PRECOG_A_COMPLEX),
                 lambda: pg.scan_inputs(x, x, torch.zeros(2, N), t[0, 0], torch.zeros(2, N), a_kind=pg.PRECOG_A_COMPLEX)):
        with pytest.raises(ValueError, match="resolve_conj"):
            take()
    plain = t.resolve_conj().resolve_neg()
    assert pg._dtype_code(plain) == pg.PRECOG_F32
    assert pg._table(plain, 8, N, torch.complex64, -1, "t") == (plain.data_ptr(), n, 1)


@pytest.mark.gpu
def test_scans_refuse_conjugated_inputs_and_states(cuda_device, pg):
    import torch
    d, n, D = cuda_device, 2, 8
    x, dt, B, C = torch.randn((4, 1, n, N), device=d)
    x, dt = x[..., :D].contiguous(), dt[..., :D].abs()
    A = torch.complex(-torch.rand((1, D, N), device=d), torch.randn((1, D, N), device=d))
    with pytest.raises(ValueError, match="resolve_conj"):
        pg.scan_inputs(x, dt, B, A.conj(), C, a_kind=pg.PRECOG_A_COMPLEX)
    h, y = torch.randn((n, 1, D, N), dtype=torch.complex64, device=d), torch.empty((1, n, D), device=d)
    inputs = pg.scan_inputs(x, dt, B, A.conj().resolve_conj(), C, a_kind=pg.PRECOG_A_COMPLEX)
    off = torch.tensor([0, 1, 2], device=d)
    for call in (lambda: pg.precog_scan_step(inputs, h.conj(), y_out=y),
                 lambda: pg.precog_prefill_from_state(inputs, n, 1, h.conj(), y_out=y),
                 lambda: pg.precog_prefill_from_state(inputs, n, 1, h, y_out=y, state_out=torch.empty_like(h).conj()),
                 lambda: pg.precog_encode_chunks(inputs, off, n, states_out=h.conj()),
                 lambda: pg.precog_encode_chunks_ordered(inputs, off, n, off[:2].clone(), states_out=h.conj())):
        with pytest.raises(ValueError, match="resolve_conj"):
            call()
    before = h.clone()
    pg.precog_scan_step(inputs, h, y_out=y)
    assert pg.precog_device_status()[0] == 0
    a, u = torch.exp(dt[0, :, :, None] * A[0].conj()), (x * dt)[0, :, :, None] * B[0, :, None, :]
    assert torch.allclose(h[:, 0], a * before[:, 0] + u, rtol=1e-5, atol=1e-5)
