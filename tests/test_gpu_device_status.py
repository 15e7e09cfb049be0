"""precog_device_status: every file's word is reported, once."""
import time

import pytest

pytestmark = pytest.mark.gpu


def test_each_word_is_reported_once(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    i64 = lambda *v: torch.tensor(v, dtype=torch.int64, device=cuda_device)  # noqa: E731
    x = torch.randn((64, 1, 64), device=cuda_device)
    g = torch.zeros((64, 1), device=cuda_device)
    none = torch.empty((64, 0, 64), device=cuda_device)
    table, y = torch.zeros((2, 1, 1, 64, 64), device=cuda_device), torch.empty((64, 1, 64), device=cuda_device)
    bf = x.to(torch.bfloat16)
    logits, out = torch.randn((1, 50), device=cuda_device), torch.empty(1, device=cuda_device)
    calls = [
        (lambda: pg.precog_delta_scan(pg.delta_inputs(None, x, x, g, g), i64(0, 65), 64, states_out=table[:1]), pg.PRECOG_DEV_BAD_OFFSETS),
        (lambda: pg.precog_delta_scan(pg.delta_inputs(None, bf, bf, g, g), i64(0, 65), 64, states_out=table[:1]), pg.PRECOG_DEV_BAD_OFFSETS),
        (lambda: pg.precog_delta_step(pg.delta_inputs(x[:1], x[:1], x[:1], g[:1], g[:1]), table, slots=i64(5), y_out=y[:1]),
         pg.PRECOG_DEV_BAD_INDEX),
        (lambda: pg.precog_qk_norm_rope(x, none, y, none, cos=torch.ones((3, 32), device=cuda_device),
                                        sin=torch.zeros((3, 32), device=cuda_device), positions=i64(*[3] * 64)), pg.PRECOG_DEV_BAD_INDEX),
        (lambda: pg.precog_token_logprobs(logits, i64(50), out), pg.PRECOG_DEV_BAD_INDEX),
        (lambda: pg.precog_selftest_wait_timeout(16), pg.PRECOG_DEV_TIMEOUT)]
    assert pg.precog_device_status() == (0, 0)
    for call, bits in calls:
        call()
        assert pg.precog_device_status()[1] == bits
        assert pg.precog_device_status() == (0, 0)


def test_asking_costs_a_launch_and_a_copy(cuda_device):
    """Not a copy for each of the library's files: less than eight of a tensor's copies to the host."""
    import torch
    import paper_2608_02560_gb300 as pg
    word, host = torch.zeros(1, dtype=torch.int32, device=cuda_device), torch.zeros(1, dtype=torch.int32)

    def best(call):
        times = []
        for _ in range(200):
            torch.cuda.synchronize()
            t = time.perf_counter()
            call()
            times.append(time.perf_counter() - t)
        return min(times)
    a, b = best(pg.precog_device_status), best(lambda: host.copy_(word))
    print(f"status {a * 1e6:.1f} us, copy {b * 1e6:.1f} us")
    assert a < 8 * b
