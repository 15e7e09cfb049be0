"""Arguments at the ends of their ranges are refused before anything is launched, or accepted."""
import pytest

FAKE = 0x10000  # an aligned address that the host never dereferences


@pytest.fixture(scope="module")
def lib():
    from paper_2608_02560_gb300 import build
    build.build()
    import paper_2608_02560_gb300 as pg
    return pg.load_library()


@pytest.mark.parametrize("temp", [2.95e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_exponent_scale_is_beyond_fp32(lib, temp):
    """log2(e) / temperature has to be finite, not 1 / temperature alone."""
    assert lib.precog_token_logprobs(FAKE, 1, 4, 100, 100, FAKE, temp, 0, FAKE, None, None, None, None) == 1
    assert b"temperature" in lib.precog_last_error()


@pytest.mark.parametrize("temp", [4.3e-39, 1e-38, 3.4e38])
def test_temperatures_at_the_ends_are_accepted(lib, temp):
    assert lib.precog_token_logprobs(FAKE, 1, 0, 100, 100, FAKE, temp, 0, FAKE, None, None, None, None) == 0
