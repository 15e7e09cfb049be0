"""Answer questions from pre-computed states of a small selective state space model.

    python examples/answer_from_scan_state.py

A layer of such a model is a short causal convolution (precog_causal_conv), a diagonal selective scan and the
end of its block (precog_block_norm: skip, gate, norm; then the residual and the next block's norm), so a
chunk leaves two things behind: the scan's state and the convolution's window. The corpus is read once and both
go into banks (precog_encode_chunks, precog_causal_conv). A question finds its chunk (precog_retrieve), starts
from that chunk's window and state (precog_causal_conv and precog_prefill_from_state with ``idx``) and is
answered token by token on the tables that this leaves (precog_conv_step, precog_scan_step). Before each choice
precog_adjust_logits penalises what the text has already and bans what the answer's grammar does not allow;
precog_token_logprobs gives the log probabilities and the likeliest tokens, of which the first is taken.

Then the same answers are scored the long way, chunk + question + answer in one scan from empty windows and
zero states: what the model gives a token does not depend on where its reading was cut.

Weights and tokens are random; the projections around the library's calls are plain torch.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_02560_gb300 as pg  # noqa: E402

VOCAB, WIDTH, INNER, LAYERS, N, K = 5003, 128, 256, 2, 16, 4


class Model:
    """A stack of selective state space layers. Projections in ``dtype``; residual, states and vectors fp32."""

    def __init__(self, dtype, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, device=device, generator=gen)  # noqa: E731
        self.dtype, self.device = dtype, device
        self.embed = rand(VOCAB, WIDTH)
        self.layers = [dict(inner=(rand(WIDTH, 2 * INNER) / WIDTH ** 0.5).to(dtype),
                            conv=0.5 * rand(INNER, K), conv_bias=0.1 * rand(INNER),
                            dt=(rand(INNER, INNER) * (0.5 / INNER ** 0.5)).to(dtype), dt_bias=rand(INNER) - 3.0,
                            B=(rand(INNER, N) * (1.0 / INNER ** 0.5)).to(dtype), C=(rand(INNER, N) / INNER ** 0.5).to(dtype),
                            A=-torch.arange(1, N + 1, device=device) * torch.exp(0.3 * rand(INNER, 1)),
                            skip=rand(INNER), norm=1.0 + 0.1 * rand(INNER),
                            out=(rand(INNER, WIDTH) / INNER ** 0.5).to(dtype), next_norm=1.0 + 0.1 * rand(WIDTH))
                       for _ in range(LAYERS)]
        self.first_norm = torch.ones(WIDTH, device=device)
        self.head = (rand(WIDTH, VOCAB) * (2.0 / WIDTH ** 0.5)).to(dtype)

    def forward(self, tokens, conv, scan):
        """``conv(layer, x, c)`` and ``scan(layer, inputs, y, skip, gate)`` advance the layer's windows and states. Where
        ``scan`` has applied skip and gate itself it says so."""
        T = tokens.numel()
        rows = lambda n: torch.empty((T, n), dtype=self.dtype, device=self.device)  # noqa: E731
        residual, x = self.embed[tokens], rows(WIDTH)
        pg.precog_block_norm(residual.to(self.dtype), out=x, weight=self.first_norm)
        for i, p in enumerate(self.layers):
            wide = x @ p["inner"]                       # the convolution's input and the gate are slices of it
            inner, gate = wide[:, :INNER], wide[:, INNER:]
            c, y, mixed = rows(INNER), rows(INNER), rows(INNER)
            conv(i, inner, c)
            dt = torch.nn.functional.softplus((c @ p["dt"]).float() + p["dt_bias"]).to(self.dtype)
            inputs = pg.scan_inputs(c, dt, c @ p["B"], p["A"], c @ p["C"])
            if scan(i, inputs, y, p["skip"], gate):
                pg.precog_block_norm(y, out=mixed, weight=p["norm"])
            else:
                pg.precog_block_norm(y, out=mixed, skip=p["skip"], skip_input=c, gate=gate, weight=p["norm"])
            pg.precog_block_norm(mixed @ p["out"], out=x, residual=residual, scale=0.7, residual_out=residual,
                                 out_weight=p["next_norm"])
        return x

    def read(self, tokens, offsets, n, length=None, windows=None, states=None, idx=None):
        """Sequences at ``offsets``, from the beginning or (all of one ``length``) from rows ``idx`` of ``windows`` and
        ``states``: the last layer's rows, the windows and states behind."""
        T = tokens.numel()
        win = torch.empty((n, LAYERS, K - 1, INNER), dtype=self.dtype, device=self.device)
        h = torch.empty((n, LAYERS, INNER, N), device=self.device)

        def conv(layer, x, c):
            p = self.layers[layer]
            pg.precog_causal_conv(x, p["conv"], offsets, bias=p["conv_bias"], bank=windows, idx=idx, layer=layer,
                                  windows_out=win, y_out=c)

        def scan(layer, inputs, y, skip, gate):
            if states is None:
                pg.precog_encode_chunks(inputs, offsets, T, states_out=h, layer0=layer, L_total=LAYERS, y_out=y[None])
            else:
                pg.precog_prefill_from_state(inputs, n, length, states, idx=idx, layer0=layer, y_out=y[None], state_out=h)

        return self.forward(tokens, conv, scan), win, h

    def step(self, tokens, windows, states):
        """One token of each row, on its slot of the tables."""
        def conv(layer, x, c):
            p = self.layers[layer]
            pg.precog_conv_step(x, p["conv"], windows, bias=p["conv_bias"], layer=layer, y_out=c)

        def scan(layer, inputs, y, skip, gate):
            pg.precog_scan_step(inputs, states, layer0=layer, skip=skip, gate=gate, y_out=y)
            return True

        return self.forward(tokens, conv, scan)


def _offsets(lens, device):
    return torch.tensor([0] + lens, device=device).cumsum(0)


def main(dtype=torch.bfloat16, answer=12, device="cuda", say=print):
    gen = torch.Generator(device=device).manual_seed(1)
    draw = lambda n: torch.randint(0, VOCAB, (n,), device=device, generator=gen)  # noqa: E731
    model = Model(dtype, device)

    # ---- once: the corpus into banks of windows and states, and its embeddings into an index
    chunk_lens = [200, 64, 131, 17, 300, 96, 1, 250]
    chunks = [draw(n) for n in chunk_lens]
    _, windows, states = model.read(torch.cat(chunks), _offsets(chunk_lens, device), len(chunks))
    index = torch.nn.functional.normalize(torch.randn((len(chunks), 64), device=device, generator=gen), dim=-1)

    # ---- questions of 24 tokens: the chunk, its windows and states, the question's own tokens
    wanted, length = [4, 0, 6, 4, 2], 24
    n = len(wanted)
    questions = [draw(length) for _ in range(n)]
    about = index[wanted] + 0.05 * torch.randn((n, 64), device=device, generator=gen)
    idx = torch.empty(n, dtype=torch.int64, device=device)
    pg.precog_retrieve(index, about, idx)
    off = _offsets([length] * n, device)
    rows, win, h = model.read(torch.cat(questions), off, n, length, windows, states, idx)
    last = rows[off[1:] - 1]

    # ---- what may be answered: two grammars, each a set of tokens; the last question has none
    bits = torch.rand((2, (VOCAB + 31) // 32, 32), device=device, generator=gen) < 0.3
    words = (bits.long() << torch.arange(32, device=device)).sum(-1)
    mask = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
    mask_rows = torch.tensor([0, 1, 1, 0, -1], device=device)
    unlikely = questions[0][:3]                          # three tokens that every answer is talked out of

    def adjust(logits, texts, grammar):
        """Penalties for what a row's question and answer have already, counted in the answer."""
        m = len(texts)
        lens = [t.numel() for t in texts]
        pg.precog_adjust_logits(
            logits, logits, history=torch.cat(texts), history_offsets=_offsets(lens, device),
            count_from=torch.full((m,), length, device=device), repetition=torch.full((m,), 1.2, device=device),
            frequency=torch.full((m,), 0.1, device=device), presence=torch.full((m,), 0.2, device=device),
            bias_idx=unlikely.repeat(m), bias=torch.full((3 * m,), -2.0, device=device),
            bias_offsets=3 * torch.arange(m + 1, device=device), mask=mask, mask_rows=grammar)

    # ---- answers, a token of every question at a time, on the tables that the prefill left
    none = torch.full((n,), -1, dtype=torch.int64, device=device)        # nothing to score: the call only chooses
    logprob = torch.empty(n, device=device)
    best, best_logprob = torch.empty((n, 5), dtype=torch.int64, device=device), torch.empty((n, 5), device=device)
    tokens, given = torch.empty((n, 0), dtype=torch.int64, device=device), []
    for _ in range(answer):
        logits = last @ model.head
        adjust(logits, [torch.cat([q, a]) for q, a in zip(questions, tokens)], mask_rows)
        pg.precog_token_logprobs(logits, none, logprob, top_idx=best, top_logprob=best_logprob)
        tokens = torch.cat([tokens, best[:, :1]], 1)
        given.append(best_logprob[:, 0].clone())
        last = model.step(best[:, 0].contiguous(), win, h)
    given = torch.stack(given, 1)

    # ---- the long way: chunk, question and answer in one scan
    found = idx.tolist()
    whole = [torch.cat([chunks[c], q, a]) for c, q, a in zip(found, questions, tokens)]
    off = _offsets([t.numel() for t in whole], device)
    rows, _, _ = model.read(torch.cat(whole), off, n)
    at = torch.cat([torch.arange(e - answer - 1, e - 1) for e in off[1:].tolist()]).to(device)
    logits = rows[at] @ model.head
    adjust(logits, [torch.cat([q, a[:j]]) for q, a in zip(questions, tokens) for j in range(answer)],
           mask_rows.repeat_interleave(answer))
    scored = torch.empty(n * answer, device=device)
    pg.precog_token_logprobs(logits, tokens.reshape(-1), scored)
    scored = scored.view(n, answer)
    status = pg.precog_device_status()

    allowed = bits.view(2, -1)[mask_rows[:-1].unsqueeze(1), tokens[:-1]]
    for i in range(n):
        say(f"question {i}: chunk {found[i]}, answer {tokens[i].tolist()}, log probability {given[i].sum():.4f}, "
            f"scored in one scan {scored[i].sum():.4f}")
    say(f"largest difference of a token's log probability: {(given - scored).abs().max():.2e}")
    return dict(found=found, wanted=wanted, tokens=tokens, given=given, scored=scored, allowed=allowed, status=status)


if __name__ == "__main__":
    result = main()
    sys.exit(0 if result["status"][0] == 0 and result["found"] == result["wanted"] else 1)
