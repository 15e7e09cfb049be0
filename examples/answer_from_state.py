"""Answer questions from pre-computed states of a small gated-delta-rule model.

    python examples/answer_from_state.py

The corpus is read once: every chunk's matrix states go into a bank (precog_delta_scan from zero
states). A question finds its chunk by embedding similarity (precog_retrieve), starts from that
chunk's states (precog_delta_scan from ``bank[idx]``) and is answered token by token
(precog_delta_step on the table of running states). precog_qk_norm_rope norms and rotates the
queries and keys of all three, and precog_token_logprobs gives the answer's log probabilities with
the likeliest tokens, of which the first is taken.

Then the same answers are scored the long way, chunk + question + answer in one scan from zero
states: what the model gives a token does not depend on where its reading was cut.

Weights and tokens are random; the projections around the library's calls are plain torch.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_02560_gb300 as pg  # noqa: E402

VOCAB, WIDTH, LAYERS, HK, HV, DK, DV, ROT = 5003, 256, 2, 2, 4, 64, 64, 32


class Model:
    """A stack of gated delta rule layers. Parameters in ``dtype``; gates, states and rotations fp32."""

    def __init__(self, dtype, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, device=device, generator=gen)  # noqa: E731
        self.dtype, self.device = dtype, device
        self.embed = rand(VOCAB, WIDTH).to(dtype)
        qkv = (2 * HK) * DK + HV * DV
        self.layers = [dict(w=(rand(WIDTH, qkv) / WIDTH ** 0.5).to(dtype),
                            gates=rand(WIDTH, 2 * HV) / WIDTH ** 0.5,
                            rate=torch.exp(rand(HV)) * 0.05,
                            out=(rand(HV * DV, WIDTH) / (HV * DV) ** 0.5).to(dtype)) for _ in range(LAYERS)]
        self.head = (rand(WIDTH, VOCAB) * (2.0 / WIDTH ** 0.5)).to(dtype)
        angle = torch.arange(4096, device=device)[:, None] * 100.0 ** (-torch.arange(ROT // 2, device=device) / (ROT // 2))
        self.cos, self.sin = torch.cos(angle), torch.sin(angle)

    def norm(self, x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(self.dtype)

    def forward(self, tokens, positions, mix):
        """``mix(layer, inputs, y)`` advances the layer's states by ``inputs`` and reads them out into ``y``."""
        x, T = self.embed[tokens], tokens.numel()
        for i, p in enumerate(self.layers):
            h = self.norm(x)
            proj = h @ p["w"]                          # q, k and v are slices of it, which the calls take as they are
            q, k, v = (t.view(T, n, d) for t, n, d in zip(proj.split([HK * DK, HK * DK, HV * DV], 1), (HK, HK, HV),
                                                          (DK, DK, DV)))
            pg.precog_qk_norm_rope(q, k, q, k, norm="l2", cos=self.cos, sin=self.sin, positions=positions)
            a, b = (h.float() @ p["gates"]).chunk(2, 1)
            inputs = pg.delta_inputs(q, k, v, -p["rate"] * torch.nn.functional.softplus(a), torch.sigmoid(b))
            y = torch.empty((T, HV, DV), dtype=self.dtype, device=self.device)
            mix(i, inputs, y)
            x = x + self.norm(y).view(T, HV * DV) @ p["out"]
        return self.norm(x)

    def scan(self, tokens, lens, starts, bank=None, idx=None):
        """Read sequences of ``lens`` whose first tokens stand at ``starts``: the last layer's rows and the states."""
        off = torch.zeros(len(lens) + 1, dtype=torch.int64, device=self.device)
        lens_t = torch.tensor(lens, device=self.device)
        off[1:] = lens_t.cumsum(0)
        T = tokens.numel()
        positions = torch.arange(T, device=self.device) + (starts - off[:-1]).repeat_interleave(lens_t, output_size=T)
        states = torch.empty((len(lens), LAYERS, HV, DV, DK), device=self.device)

        def mix(layer, inputs, y):
            pg.precog_delta_scan(inputs, off, T, bank=bank, idx=idx, layer=layer, states_out=states, y_out=y)

        return self.forward(tokens, positions, mix), states, off


def main(dtype=torch.bfloat16, answer=12, device="cuda", say=print):
    gen = torch.Generator(device=device).manual_seed(1)
    draw = lambda n: torch.randint(0, VOCAB, (n,), device=device, generator=gen)  # noqa: E731
    model = Model(dtype, device)

    # ---- once: the corpus into a bank of states, and its embeddings into an index
    chunk_lens = [200, 64, 131, 17, 300, 96, 1, 250]
    chunks = [draw(n) for n in chunk_lens]
    zero = torch.zeros(len(chunks), dtype=torch.int64, device=device)
    _, bank, _ = model.scan(torch.cat(chunks), chunk_lens, zero)
    index = torch.nn.functional.normalize(torch.randn((len(chunks), 64), device=device, generator=gen), dim=-1)

    # ---- questions: the chunk, its states, the question's own tokens
    wanted, lens = [4, 0, 6, 4, 2], [9, 30, 64, 1, 70]
    n = len(lens)
    questions = [draw(m) for m in lens]
    about = index[wanted] + 0.05 * torch.randn((n, 64), device=device, generator=gen)
    idx = torch.empty(n, dtype=torch.int64, device=device)
    pg.precog_retrieve(index, about, idx)
    starts = torch.tensor(chunk_lens, device=device)[idx]
    rows, states, off = model.scan(torch.cat(questions), lens, starts, bank, idx)

    # ---- answers, a token of every question at a time, on the states that the prefill left
    token = torch.full((n,), -1, dtype=torch.int64, device=device)      # the first call only chooses
    logprob, entropy = torch.empty(n, device=device), torch.empty(n, device=device)
    best, best_logprob = torch.empty((n, 5), dtype=torch.int64, device=device), torch.empty((n, 5), device=device)
    last, positions = rows[off[1:] - 1], starts + torch.tensor(lens, device=device)

    def mix(layer, inputs, y):
        pg.precog_delta_step(inputs, states, y_out=y, layer=layer)

    given, tokens, entropies = [], [], []
    for _ in range(answer):
        pg.precog_token_logprobs(last @ model.head, token, logprob, entropy, best, best_logprob)
        token = best[:, 0].clone()
        tokens.append(token)
        given.append(best_logprob[:, 0].clone())
        entropies.append(entropy.clone())
        last, positions = model.forward(token, positions, mix), positions + 1
        token = torch.full_like(token, -1)
    tokens, given, entropies = (torch.stack(t, 1) for t in (tokens, given, entropies))

    # ---- the long way: chunk, question and answer in one scan
    found = idx.tolist()
    whole = [torch.cat([chunks[c], q, a]) for c, q, a in zip(found, questions, tokens)]
    whole_lens = [t.numel() for t in whole]
    rows, _, off = model.scan(torch.cat(whole), whole_lens, zero[:n])
    at = torch.cat([torch.arange(e - answer - 1, e - 1) for e in off[1:].tolist()]).to(device)
    scored = torch.empty(n * answer, device=device)
    pg.precog_token_logprobs(rows[at] @ model.head, tokens.reshape(-1), scored)
    scored = scored.view(n, answer)
    status = pg.precog_device_status()

    for i in range(n):
        say(f"question {i}: chunk {found[i]}, answer {tokens[i].tolist()}, log probability {given[i].sum():.4f}, "
            f"scored in one scan {scored[i].sum():.4f}")
    say(f"largest difference of a token's log probability: {(given - scored).abs().max():.2e}")
    return dict(found=found, wanted=wanted, tokens=tokens, given=given, scored=scored, entropy=entropies, status=status)


if __name__ == "__main__":
    result = main()
    sys.exit(0 if result["status"][0] == 0 and result["found"] == result["wanted"] else 1)
