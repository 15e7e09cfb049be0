"""Complex rows are not fp32 rows: where the header says F32, BF16 or F16 the calls take real tensors (a complex64
tensor's memory is twice as many numbers). Banks and tables of states are the only complex ones."""
import pytest

N = 16


@pytest.fixture(scope="module")
def pg():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg


def test_complex_rows_are_refused(pg, monkeypatch):
    import torch
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    z = torch.zeros(6, 8, dtype=torch.complex64)
    x, w, off = torch.zeros(6, 8), torch.zeros(8, 4), torch.tensor([0, 6])
    hand = pg.ScanInputs(1, 8, N, pg.PRECOG_F32, pg.PRECOG_A_GENERAL, 0, 16, 16, 16, 16, 16, 48, 96)
    hand.rows, hand.device, hand._keepalive = 6, -1, (x,)
    B, A, h = torch.zeros(6, N), torch.zeros(8, N), torch.zeros(6, 1, 8, N)
    for call in (lambda: pg.precog_causal_conv(z, w, off, y_out=z.clone()),
                 lambda: pg.precog_conv_step(z, w, torch.zeros(6, 1, 3, 8, dtype=torch.complex64), y_out=z.clone()),
                 lambda: pg.precog_block_norm(z, out=z.clone()),
                 lambda: pg.precog_block_norm(x, residual=z, residual_out=z.clone()),
                 lambda: pg.precog_adjust_logits(z, z.clone()),
                 lambda: pg.precog_scan_step(hand, h, y_out=z[None].clone()),
                 lambda: pg.scan_inputs(z, z, B.to(z.dtype), A, B.to(z.dtype)),
                 lambda: pg._row_code(z)):
        with pytest.raises(TypeError, match="complex64"):
            call()
