"""Rows, weights and masks that are no matrices are refused by name (not by Python's unpacking or indexing)."""
import pytest


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


@pytest.mark.parametrize("shape", [(8,), (2, 3, 8), ()])
def test_rows_are_matrices(on_host, shape):
    import torch
    pg, bad = on_host, torch.zeros(shape)
    w, off, win = torch.zeros(8, 4), torch.tensor([0, 2]), torch.zeros(2, 1, 3, 8)
    for call in (lambda: pg.precog_causal_conv(bad, w, off, y_out=bad), lambda: pg.precog_conv_step(bad, w, win, y_out=bad),
                 lambda: pg.precog_block_norm(bad, out=bad)):
        with pytest.raises(ValueError, match="x must be"):
            call()
    with pytest.raises(ValueError, match="logits must be"):
        pg.precog_adjust_logits(bad, bad)


@pytest.mark.parametrize("shape", [(), (8,), (8, 4, 1), (9, 4)])
def test_weights_are_matrices_of_the_rows_channels(on_host, shape):
    import torch
    x, y = torch.zeros(6, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError, match="weight must be"):
        on_host.precog_causal_conv(x, torch.zeros(shape), torch.tensor([0, 6]), y_out=y)
    with pytest.raises(ValueError, match="weight must be"):
        on_host.precog_conv_step(x, torch.zeros(shape), torch.zeros(6, 1, 3, 8), y_out=y)


def test_masks_are_matrices(on_host):
    import torch
    x, y = torch.zeros(3, 8), torch.zeros(3, 8)
    for shape in ((), (3,), (3, 1, 1)):
        with pytest.raises(ValueError, match="mask must be"):
            on_host.precog_adjust_logits(x, y, mask=torch.zeros(shape, dtype=torch.int32))
