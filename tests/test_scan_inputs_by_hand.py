"""A ScanInputs that was filled field by field, without scan_inputs, serves precog_scan_step as it does the other scans."""
import pytest

N = 16


@pytest.fixture(scope="module")
def pg():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg


@pytest.fixture
def on_host(pg, monkeypatch):
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    monkeypatch.setattr(pg, "_stream_on", lambda device, stream: None)
    return pg


def _by_hand(pg, x, dt, B, A, C):
    L, n, D = x.shape
    return pg.ScanInputs(L, D, N, pg._row_code(x), pg.PRECOG_A_GENERAL, 0, x.data_ptr(), dt.data_ptr(), B.data_ptr(),
                         C.data_ptr(), A.data_ptr(), n * D, n * N)


def test_a_step_checks_its_arguments_against_inputs_filled_by_hand(on_host):
    import torch
    pg, (x, dt), (B, C), A = on_host, torch.zeros(2, 2, 3, 8), torch.zeros(2, 2, 3, N), torch.zeros(2, 8, N)
    hand, h, y = _by_hand(pg, x, dt, B, A, C), torch.zeros(3, 2, 8, N), torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="y_out"):
        pg.precog_scan_step(hand, h)
    with pytest.raises(ValueError, match="y_out must be"):
        pg.precog_scan_step(hand, h, y_out=y[0])
    with pytest.raises(ValueError, match="y_out must be"):
        pg.precog_scan_step(hand, h, y_out=y[:1])
    with pytest.raises(ValueError, match="gate must be"):
        pg.precog_scan_step(hand, h, gate=y[:, :2], y_out=y)
    with pytest.raises(TypeError, match="gate"):
        pg.precog_scan_step(hand, h, gate=y.bfloat16(), y_out=y)
    with pytest.raises(ValueError, match="slots must be"):
        pg.precog_scan_step(hand, h, slots=torch.zeros(2, dtype=torch.int64), y_out=y)


@pytest.mark.gpu
def test_a_step_of_inputs_filled_by_hand(cuda_device, pg):
    import torch
    d, L, n, D = cuda_device, 2, 5, 64
    x, dt, B, C = torch.randn((L, n, D), device=d), torch.rand((L, n, D), device=d), torch.randn((L, n, N), device=d), torch.randn((L, n, N), device=d)
    A, h, gate = -torch.rand((L, D, N), device=d), torch.randn((n, L, D, N), device=d), torch.randn((L, n, D), device=d)
    states, out = [], []
    for inputs in (pg.scan_inputs(x, dt, B, A, C), _by_hand(pg, x, dt, B, A, C)):
        states.append(h.clone())
        out.append(torch.empty((L, n, D), device=d))
        pg.precog_scan_step(inputs, states[-1], gate=gate, y_out=out[-1])
    assert pg.precog_device_status()[0] == 0
    assert torch.equal(*states) and torch.equal(*out)
