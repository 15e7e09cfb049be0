"""Grammar masks with nothing in them. torch gives an empty tensor the address 0, which the C call reads as "no masks":
rows that have none to go by are refused, not allowed every token."""
import ctypes

import pytest

FAKE = 0x10000000  # a 16-byte aligned address that the host never dereferences


@pytest.fixture(scope="module")
def pg():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg


@pytest.mark.parametrize("masks", [0, 2])
def test_fewer_masks_than_rows(pg, monkeypatch, masks):
    import torch
    monkeypatch.setattr(pg, "_current_device", lambda: -1)     # (a host tensor's)
    monkeypatch.setattr(pg, "_stream_on", lambda device, stream: None)
    x, out, mask = torch.zeros(3, 50), torch.zeros(3, 50), torch.zeros((masks, 2), dtype=torch.int32)
    with pytest.raises((ValueError, pg.PrecogError), match="fewer masks than rows"):
        pg.precog_adjust_logits(x, out, mask=mask)
    pg.precog_adjust_logits(x[:0], out[:0], mask=mask)


def test_masks_that_are_counted_have_an_address(pg):
    a = pg.AdjustArgs(dtype=pg.PRECOG_BF16, vocab=100, stride=100, out_stride=100, logits=FAKE, out=FAKE + (1 << 24), n_masks=4)
    assert pg.load_library().precog_adjust_logits(ctypes.byref(a), 4, None) == 1
