"""Batches of no rows are answered without a launch. torch gives an empty tensor the address 0, which is no reason to
refuse it: the tables of a server between two requests, the last part of a corpus."""
import pytest

N = 16


@pytest.fixture
def pg(monkeypatch):
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    monkeypatch.setattr(pg, "_stream_on", lambda device, stream: None)
    before = pg.load_library().precog_launch_count()
    yield pg
    assert pg.load_library().precog_launch_count() == before


@pytest.mark.parametrize("residual", [False, True])
def test_block_norm(pg, residual):
    import torch
    rows, vec = torch.zeros(0, 64), torch.zeros(64)
    more = dict(residual=rows, residual_out=rows) if residual else {}
    pg.precog_block_norm(rows, out=rows, skip=vec, skip_input=rows, gate=rows, weight=vec, **more)


def test_adjusted_logits(pg):
    import torch
    pg.precog_adjust_logits(torch.zeros(0, 64), torch.zeros(0, 64), mask=torch.zeros((0, 2), dtype=torch.int32))


@pytest.mark.parametrize("slots", [0, 5])
def test_convolutions(pg, slots):
    import torch
    rows, w = torch.zeros(0, 64), torch.zeros(64, 4)
    pg.precog_conv_step(rows, w, torch.zeros(slots, 2, 3, 64), y_out=rows)
    pg.precog_causal_conv(rows, w, torch.tensor([0]), bank=torch.zeros(slots, 2, 3, 64), windows_out=torch.zeros(0, 2, 3, 64), y_out=rows)


@pytest.mark.parametrize("slots", [0, 5])
def test_scan_step(pg, slots):
    import torch
    rows, A = torch.zeros(1, 0, 64), torch.zeros(1, 64, N)
    inputs = pg.ScanInputs(1, 64, N, pg.PRECOG_F32, pg.PRECOG_A_GENERAL, 0, 0, 0, 0, 0, A.data_ptr(), 0, 0)
    inputs.rows, inputs.device, inputs._keepalive = 0, -1, (rows, A)
    pg.precog_scan_step(inputs, torch.zeros(slots, 2, 64, N), skip=torch.zeros(1, 64), gate=rows, y_out=rows)


def test_what_is_wrong_without_rows_too(pg):
    import torch
    rows = torch.zeros(0, 64)
    for call in (lambda: pg.precog_conv_step(rows, torch.zeros(64, 4), torch.zeros(0, 2, 3, 64), layer=2, y_out=rows),
                 lambda: pg.precog_block_norm(rows, out=rows, groups=3), lambda: pg.precog_block_norm(rows, out=rows, eps=-1.0)):
        with pytest.raises(pg.PrecogError):
            call()
