"""A token through a layer (convolution, scan, block norms, adjusted logits, log probabilities), captured once and
replayed on refilled inputs and advancing tables, gives the bits of the same calls made eagerly; two captures that
are replayed on two streams at once do not meet; and calls on a stream that is given run on it."""
import pytest

pytestmark = pytest.mark.gpu
N = 16


class Layer:
    def __init__(self, dev, seed, n=37, D=264, V=1003, T=90):
        import torch
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.rn = rn = lambda *s: torch.randn(s, device=dev, generator=gen)  # noqa: E731
        self.gen, self.dev, self.n, self.D, self.V = gen, dev, n, D, V
        bf = torch.bfloat16
        self.prompt, self.offsets = rn(T, D).to(bf), torch.tensor([0, 1, 40, 40, T], device=dev)
        self.bank, self.bank_idx = rn(6, 1, 3, D).to(bf), torch.tensor([5, -1, 0, 2], device=dev)
        self.x, self.gate, self.dt = rn(n, D).to(bf), rn(n, D).to(bf), rn(n, D).abs().to(bf)
        self.B, self.C, self.A = rn(n, N).to(bf), rn(n, N).to(bf), -rn(D, N).abs()
        self.w, self.b, self.skip, self.weight = rn(D, 4), rn(D), rn(1, D), rn(D)
        self.slots = torch.randperm(n + 3, device=dev, generator=gen)[:n].contiguous()
        self.head = rn(D, V).to(bf)
        self.history = torch.randint(0, V, (n * 20,), device=dev, generator=gen)
        self.h_off, self.rep = 20 * torch.arange(n + 1, device=dev), 1.0 + rn(n).abs()
        self.mask = torch.randint(-2 ** 31, 2 ** 31, (2, (V + 31) // 32), device=dev, generator=gen).int()
        self.rows = torch.arange(n, device=dev) % 3 - 1
        self.windows, self.states = rn(n + 3, 1, 3, D).to(bf), rn(n + 3, 1, D, N)
        self.residual = rn(n, D)

    def refill(self):
        for t in (self.x, self.gate, self.B, self.C, self.prompt, self.bank):
            t.copy_(self.rn(*t.shape))

    def outputs(self):
        import torch
        e = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device=self.dev)  # noqa: E731
        return dict(py=e(*self.prompt.shape), pw=e(4, 1, 3, self.D), c=e(self.n, self.D), y=e(1, self.n, self.D),
                    m=e(self.n, self.D), o=e(self.n, self.D), z=e(self.n, self.V), lp=e(self.n, dtype=torch.float32),
                    best=e(self.n, 3, dtype=torch.int64), best_lp=e(self.n, 3, dtype=torch.float32))

    def run(self, o, stream=None):
        import torch
        import paper_2608_02560_gb300 as pg
        pg.precog_causal_conv(self.prompt, self.w, self.offsets, bias=self.b, bank=self.bank, idx=self.bank_idx,
                              windows_out=o["pw"], y_out=o["py"], stream=stream)
        pg.precog_conv_step(self.x, self.w, self.windows, slots=self.slots, bias=self.b, y_out=o["c"], stream=stream)
        pg.precog_scan_step(pg.scan_inputs(o["c"], self.dt, self.B, self.A, self.C), self.states, slots=self.slots,
                            skip=self.skip, gate=self.gate, y_out=o["y"], stream=stream)
        pg.precog_block_norm(o["y"][0], out=o["m"], weight=self.weight, stream=stream)
        pg.precog_block_norm(o["m"], out=o["o"], residual=self.residual, residual_out=self.residual, scale=0.5,
                             out_weight=self.weight, stream=stream)
        if stream is None:
            torch.mm(o["o"], self.head, out=o["z"])
        else:
            with torch.cuda.stream(stream):
                torch.mm(o["o"], self.head, out=o["z"])
        pg.precog_adjust_logits(o["z"], o["z"], history=self.history, history_offsets=self.h_off, repetition=self.rep,
                                mask=self.mask, mask_rows=self.rows, stream=stream)
        pg.precog_token_logprobs(o["z"], self.history[:self.n], o["lp"], top_idx=o["best"], top_logprob=o["best_lp"],
                                 stream=stream)

    def tables(self):
        return {"windows": self.windows, "states": self.states, "residual": self.residual}


def _same(a, b):
    import torch
    assert a.keys() == b.keys()
    for k in a:
        assert torch.equal(torch.nan_to_num(a[k].float(), 5.0), torch.nan_to_num(b[k].float(), 5.0)), k


def _captured(layer):
    import torch
    out, side, g = layer.outputs(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    held = {k: v.clone() for k, v in layer.tables().items()}
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run(out)
    torch.cuda.current_stream().wait_stream(side)
    for k, v in layer.tables().items():
        v.copy_(held[k])
    with torch.cuda.graph(g):
        layer.run(out)
    return g, out


def test_captured_tokens_are_the_eager_ones(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    eager, layer = Layer(cuda_device, 1), Layer(cuda_device, 1)
    g, out = _captured(layer)
    plain = eager.outputs()
    for _ in range(3):
        eager.refill(), layer.refill()
        eager.run(plain)
        g.replay()
        torch.cuda.synchronize()
        _same(plain, out)
        _same(eager.tables(), layer.tables())
    assert pg.precog_device_status()[0] == 0


def test_two_graphs_on_two_streams_do_not_meet(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    layers, alone = [Layer(cuda_device, s) for s in (2, 3)], [Layer(cuda_device, s) for s in (2, 3)]
    graphs = [_captured(layer) for layer in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for layer, (_, out), other in zip(layers, graphs, alone):
        plain = other.outputs()
        for _ in range(5):
            other.run(plain)
        torch.cuda.synchronize()
        _same(plain, out)
        _same(other.tables(), layer.tables())
    assert pg.precog_device_status()[0] == 0


def test_a_given_stream_is_the_one_that_is_used(cuda_device):
    import torch
    layer, other = Layer(cuda_device, 4), Layer(cuda_device, 4)
    s, out, plain = torch.cuda.Stream(), layer.outputs(), other.outputs()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)            # the tokens' inputs arrive late on that stream
        layer.x.mul_(2.0)
    layer.run(out, stream=s)
    other.x.mul_(2.0)
    other.run(plain)
    torch.cuda.synchronize()
    _same(plain, out)
    _same(other.tables(), layer.tables())


def test_tensors_of_another_device_are_refused(cuda_device, monkeypatch):
    import torch
    import paper_2608_02560_gb300 as pg
    layer = Layer(cuda_device, 5)
    out = layer.outputs()
    monkeypatch.setattr(pg, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        layer.run(out)
    torch.cuda.synchronize()
