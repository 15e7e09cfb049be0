"""The operators around a matrix-valued recurrent state, as timed and compared cases.

Kinds of case (``case["op"]``):

* ``delta``    -- the gated delta rule over a ragged batch of token sequences: chunks encoded
  into a bank of states, or queries prefilled from retrieved states with a readout a token;
* ``step``     -- the same recurrence for one token of each sequence of a serving batch, on a
  table of fp32 states that is updated in place;
* ``qk``       -- the norm of each query and key head with the position rotation;
* ``logprobs`` -- log probabilities of given tokens, entropy, and the best alternatives.

Shapes: q, k ``[T, Hk, dk]``, v ``[T, Hv, dv]``, gates ``g`` (log decay) and ``beta``
``[T, Hv]`` fp32, states ``[entries, layers, Hv, dv, dk]``; value head h reads q/k head
h // (Hv / Hk).
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"
CHUNK = 64


def listed():
    return [
        # One user's question of 64 tokens, prefilled from the state that the retrieval chose
        # (a bf16 bank), the state kept in fp32 for the answer's tokens: a call's latency.
        dict(name="delta_query_one", op="delta", n=1, least=64, most=64, hk=8, hv=16, dk=128, dv=128, dtype="bf16",
             y="bf16", out="f32", bank="bf16", entries=16, layers=2, layer=1),
        # A server's batch of questions of odd lengths, each from its own retrieved state.
        dict(name="delta_query_batch", op="delta", n=96, least=1, most=200, hk=8, hv=16, dk=128, dv=128, dtype="bf16",
             y="bf16", out="f32", bank="bf16", entries=64, layers=2, layer=0),
        # Bulk indexing of a ragged corpus: states captured into a bf16 bank, no readout.
        dict(name="delta_encode_corpus", op="delta", n=256, least=256, most=4096, hk=4, hv=8, dk=128, dv=128,
             dtype="bf16", y="none", out="bf16", bank="none", entries=0, layers=1, layer=0),
        # One long document read with its readout (scoring): little to run at once, a long axis.
        dict(name="delta_long_one", op="delta", n=1, least=32768, most=32768, hk=8, hv=16, dk=128, dv=128,
             dtype="bf16", y="bf16", out="f32", bank="none", entries=0, layers=1, layer=0),
        # The small exact check: fp32 throughout, eight chunks of up to 256 tokens.
        dict(name="delta_f32_small", op="delta", n=8, least=129, most=256, hk=4, hv=4, dk=64, dv=64, dtype="f32",
             y="f32", out="f32", bank="f32", entries=8, layers=1, layer=0),
        # One answer token of one user: the smallest call.
        dict(name="step_one", op="step", n=1, slots=4, hk=8, hv=16, dk=128, dv=128, dtype="bf16", y="bf16", layers=1,
             layer=0),
        # One token of each of 256 users' answers: the states pass through memory once.
        dict(name="step_batch", op="step", n=256, slots=300, hk=8, hv=16, dk=128, dv=128, dtype="bf16", y="bf16",
             layers=1, layer=0),
        # Queries and keys of one decoded token, as slices of a fused projection.
        dict(name="qk_one", op="qk", tokens=1, hq=16, hk=8, d=128, rot=64, norm="l2", dtype="bf16", inter=False,
             weight=False, positions=4096),
        # Queries and keys of a corpus batch, RMS norm with weights, the whole head rotated.
        dict(name="qk_corpus", op="qk", tokens=65521, hq=16, hk=8, d=128, rot=128, norm="rms", dtype="bf16",
             inter=True, weight=True, positions=32768),
        # The next token of one answer: a single row of logits with five alternatives.
        dict(name="logprobs_one", op="logprobs", rows=1, vocab=32000, pad=0, dtype="bf16", k=5, banned=0.0, temp=1.0),
        # Scoring the answers of a batch: every position's token over an odd vocabulary.
        dict(name="logprobs_score", op="logprobs", rows=2048, vocab=50257, pad=0, dtype="bf16", k=5, banned=0.0,
             temp=1.0),
        # A decoding batch in fp32, most tokens banned by a grammar, at a temperature.
        dict(name="logprobs_banned", op="logprobs", rows=61, vocab=128001, pad=7, dtype="f32", k=20, banned=0.9,
             temp=0.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["delta", "delta", "delta", "step", "qk", "logprobs"])
    if op in ("delta", "step"):
        hk = _log(rng, 1, 16)
        c = dict(op=op, hk=hk, hv=hk * rng.choice([1, 2, 4]), dk=rng.choice([64, 128, 8 * rng.randint(1, 16)]),
                 dv=rng.choice([64, 128, 8 * rng.randint(1, 32)]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        c["layers"] = rng.randint(1, 3)
        c["layer"] = rng.randrange(c["layers"])
        if op == "step":
            c["n"] = _log(rng, 1, 256)
            c["slots"] = c["n"] + rng.randint(0, 50)
            c["y"] = c["dtype"]
            return c
        c["n"] = _log(rng, 1, 128)
        most = _log(rng, 1, 8192)
        # at most about the work of the corpus case, a quarter of it in fp32 (which the
        # matrix instructions of 16 bits do not serve)
        cap = 2.0e10 if c["dtype"] == "bf16" else 1.0e9
        most = max(1, min(most, int(cap / (c["n"] * c["hv"] * c["dk"] * c["dv"]))))
        c["most"], c["least"] = most, rng.randint(0, most)
        kind = rng.choice(["encode", "query", "query"])
        c["entries"] = 0 if kind == "encode" else rng.randint(1, 2 * c["n"])
        c["bank"] = "none" if kind == "encode" else rng.choice(["bf16", "f32"])
        c["y"] = "none" if kind == "encode" else c["dtype"]
        c["out"] = rng.choice(["bf16", "f32"])
        return c
    if op == "qk":
        d = rng.choice([64, 128, 8 * rng.randint(2, 32)])
        return dict(op=op, tokens=_log(rng, 1, 40000), hq=_log(rng, 1, 32), hk=_log(rng, 1, 8), d=d,
                    rot=2 * rng.randint(0, d // 2), norm=rng.choice(["l2", "rms", "none"]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), inter=rng.random() < 0.5, weight=rng.random() < 0.5,
                    positions=_log(rng, 1, 32768))
    vocab = _log(rng, 100, 152000)
    return dict(op=op, rows=max(1, min(_log(rng, 1, 2048), int(1.0e8 / vocab))), vocab=vocab, pad=rng.randint(0, 9),
                dtype=rng.choice(["bf16", "f32", "f16"]), k=rng.randint(0, min(20, vocab)),
                banned=rng.choice([0.0, 0.0, 0.5, 0.95]), temp=rng.choice([1.0, 1.0, 0.6, 1.3]))


def _lens(case, seed):
    """The case's lengths, in an order of the seed's (so that every seed has as many tokens)."""
    r = random.Random(13)
    lens = [r.randint(case["least"], case["most"]) for _ in range(case["n"])]
    if sum(lens) == 0:
        lens[0] = 1
    random.Random(int(seed)).shuffle(lens)
    return lens


def _gates(gen, T, hv):
    """log decays -rate_h * softplus(z - 2) with rates over two orders, beta = sigmoid."""
    z = torch.randn((T, hv), device=DEV, generator=gen)
    rate = torch.exp(torch.empty(hv, device=DEV).uniform_(math.log(0.03), math.log(3.0), generator=gen))
    g = -rate * torch.nn.functional.softplus(z - 2.0)
    return g, torch.sigmoid(torch.randn((T, hv), device=DEV, generator=gen))


def _qkv(gen, T, hk, hv, dk, dv, dt):
    unit = lambda x: (x / x.square().sum(-1, keepdim=True).add(1e-6).sqrt()).to(dt)  # noqa: E731
    q = unit(torch.randn((T, hk, dk), device=DEV, generator=gen))
    k = unit(torch.randn((T, hk, dk), device=DEV, generator=gen))
    return q, k, torch.randn((T, hv, dv), device=DEV, generator=gen).to(dt)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1009 + 17)
    c, dt = dict(case), DTYPES[case["dtype"]]
    s = {"case": c}
    if c["op"] == "delta":
        lens = _lens(c, seed)
        T = sum(lens)
        s["lens"], s["T"] = lens, T
        off = [0]
        for n in lens:
            off.append(off[-1] + n)
        s["offsets"] = torch.tensor(off, dtype=torch.int64, device=DEV)
        s["q"], s["k"], s["v"] = _qkv(gen, T, c["hk"], c["hv"], c["dk"], c["dv"], dt)
        s["g"], s["beta"] = _gates(gen, T, c["hv"])
        shape = (c["layers"], c["hv"], c["dv"], c["dk"])
        s["bank"] = s["idx"] = None
        if c["bank"] != "none":
            s["bank"] = (0.3 * torch.randn((c["entries"],) + shape, device=DEV, generator=gen)).to(DTYPES[c["bank"]])
            # retrieved rows; -1 where nothing was comparable
            s["idx"] = torch.randint(-1, c["entries"], (c["n"],), device=DEV, generator=gen)
        s["states"] = torch.zeros((c["n"],) + shape, dtype=DTYPES[c["out"]], device=DEV)
        s["y"] = None if c["y"] == "none" else torch.zeros((T, c["hv"], c["dv"]), dtype=DTYPES[c["y"]], device=DEV)
    elif c["op"] == "step":
        s["q"], s["k"], s["v"] = _qkv(gen, c["n"], c["hk"], c["hv"], c["dk"], c["dv"], dt)
        s["g"], s["beta"] = _gates(gen, c["n"], c["hv"])
        s["states"] = 0.3 * torch.randn((c["slots"], c["layers"], c["hv"], c["dv"], c["dk"]), device=DEV, generator=gen)
        s["slots"] = torch.randperm(c["slots"], device=DEV, generator=gen)[:c["n"]].contiguous()
        s["y"] = torch.zeros((c["n"], c["hv"], c["dv"]), dtype=DTYPES[c["y"]], device=DEV)
    elif c["op"] == "qk":
        T, hq, hk, d = c["tokens"], c["hq"], c["hk"], c["d"]
        proj = torch.randn((T, (hq + 2 * hk) * d), device=DEV, generator=gen).to(dt)
        s["q"] = proj[:, :hq * d].view(T, hq, d)
        s["k"] = proj[:, hq * d:(hq + hk) * d].view(T, hk, d)
        s["wq"] = s["wk"] = s["cos"] = s["sin"] = s["pos"] = None
        if c["weight"]:
            s["wq"], s["wk"] = (1.0 + 0.2 * torch.randn((2, d), device=DEV, generator=gen)).unbind(0)
        if c["rot"]:
            freq = 10000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"])
            angle = torch.arange(c["positions"], device=DEV, dtype=torch.float64)[:, None] * freq
            s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
            s["pos"] = torch.randint(0, c["positions"], (T,), device=DEV, generator=gen)
        s["q_out"], s["k_out"] = (torch.zeros((T, h, d), dtype=dt, device=DEV) for h in (hq, hk))
    else:
        R, V = c["rows"], c["vocab"]
        x = 2.5 * torch.randn((R, V + c["pad"]), device=DEV, generator=gen)
        if c["banned"]:
            x.masked_fill_(torch.rand((R, V + c["pad"]), device=DEV, generator=gen) < c["banned"], -math.inf)
            x[:, 0] = 1.0                      # the end token is never banned
        s["logits"] = x.to(dt)[:, :V]
        s["tokens"] = torch.randint(0, V, (R,), device=DEV, generator=gen)
        s["logprob"], s["entropy"] = (torch.zeros(R, device=DEV) for _ in range(2))
        s["top_idx"] = torch.zeros((R, c["k"]), dtype=torch.int64, device=DEV) if c["k"] else None
        s["top_logprob"] = torch.zeros((R, c["k"]), device=DEV) if c["k"] else None
    return s


# ------------------------------------------------------------------------------ plain forms


def _heads(x, hv):
    """[..., Hk, d] -> [..., Hv, d]: each q/k head once for every value head of its group."""
    return x.repeat_interleave(hv // x.shape[-2], dim=-2)


def _start_states(s, dtype):
    c = s["case"]
    if s["bank"] is None:
        return torch.zeros((c["n"], c["hv"], c["dv"], c["dk"]), dtype=dtype, device=DEV)
    got = s["bank"][s["idx"].clamp(min=0), c["layer"]].to(dtype)
    return got * (s["idx"] >= 0).to(dtype)[:, None, None, None]


def _plain_delta(s):
    """The chunked form: 64 tokens of every sequence a pass. Chunks follow one another by
    definition (each begins with the state that the one before it leaves): hence the loop."""
    c = s["case"]
    hv, want_y = c["hv"], s["y"] is not None
    scale = c["dk"] ** -0.5
    first, last = s["offsets"][:-1, None], s["offsets"][1:, None]
    S = _start_states(s, torch.float32).transpose(-1, -2).contiguous()          # [n, Hv, dk, dv]
    y = torch.zeros((s["T"] + 1, hv, c["dv"]), device=DEV) if want_y else None   # the last row: nobody's
    low = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device=DEV).tril()
    eye = torch.eye(CHUNK, device=DEV)
    for at in range(0, max(s["lens"]), CHUNK):
        rows = first + at + torch.arange(CHUNK, device=DEV)
        there = rows < last                                                     # [n, 64]
        take = rows.clamp(max=s["T"] - 1)
        valid = there[:, None, :, None]
        k = _heads(s["k"][take].float(), hv).transpose(1, 2) * valid            # [n, Hv, 64, dk]
        v = s["v"][take].float().transpose(1, 2)
        beta = s["beta"][take].transpose(1, 2)[..., None] * valid
        b = (s["g"][take].transpose(1, 2) * there[:, None, :]).cumsum(-1)[..., None]
        decay = torch.exp((b - b.transpose(-1, -2)).masked_fill(~low, -math.inf))
        A = (beta * (k @ k.transpose(-1, -2)) * decay).tril(-1)
        inv, power = eye - A, A @ A                                             # (I + A)^-1, A nilpotent
        for _ in range(5):
            inv, power = inv + inv @ power, power @ power
        u = inv @ (beta * (v - torch.exp(b) * (k @ S)))
        if want_y:
            q = _heads(s["q"][take].float(), hv).transpose(1, 2)
            o = scale * (torch.exp(b) * (q @ S) + ((q @ k.transpose(-1, -2)) * decay) @ u)
            y[torch.where(there, rows, s["T"])] = o.transpose(1, 2)
        end = b[..., -1:, :]
        S = torch.exp(end) * S + (torch.exp(end - b) * k).transpose(-1, -2) @ u
    s["states"][:, c["layer"]] = S.transpose(-1, -2).to(s["states"].dtype)
    return {"y": y[:-1].to(s["y"].dtype) if want_y else None, "states": s["states"]}


def _plain_step(s):
    c = s["case"]
    hv = c["hv"]
    q, k = _heads(s["q"].float(), hv), _heads(s["k"].float(), hv)
    S = s["states"][s["slots"], c["layer"]] * torch.exp(s["g"])[..., None, None]
    u = s["beta"][..., None] * (s["v"].float() - (S * k[:, :, None, :]).sum(-1))
    S = S + u[..., None] * k[:, :, None, :]
    s["states"][s["slots"], c["layer"]] = S
    y = c["dk"] ** -0.5 * (S * q[:, :, None, :]).sum(-1)
    return {"y": y.to(s["y"].dtype), "states": s["states"]}


def _plain_qk_one(x, w, s):
    c = s["case"]
    x = x.float()
    if c["norm"] != "none":
        total = x.square().sum(-1, keepdim=True)
        x = x * torch.rsqrt((total if c["norm"] == "l2" else total / c["d"]) + 1e-6)
    if w is not None:
        x = x * w
    if c["rot"]:
        half = c["rot"] // 2
        cos, sin = s["cos"][s["pos"]][:, None], s["sin"][s["pos"]][:, None]
        a, b = (x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2]) if c["inter"] else (x[..., :half], x[..., half:c["rot"]])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack((a, b), -1).flatten(-2) if c["inter"] else torch.cat((a, b), -1)
        x = torch.cat((turned, x[..., c["rot"]:]), -1)
    return x.to(s["q"].dtype)


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float() / c["temp"]
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    p /= total
    logp = z - lse
    entropy = -(p * logp.masked_fill(p == 0, 0.0)).sum(-1)
    out = {"logprob": logp.gather(1, s["tokens"][:, None])[:, 0], "entropy": entropy}
    if c["k"]:
        # ordered bits above, the complement of the index below: ties to the lowest index
        bits = (s["logits"].float() + 0.0).contiguous().view(torch.int32).to(torch.int64)
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = order * (1 << 20) + ((1 << 20) - 1 - torch.arange(c["vocab"], device=DEV))
        best = torch.topk(key, c["k"], dim=-1).values
        out["top_idx"] = (1 << 20) - 1 - (best & ((1 << 20) - 1))
        out["top_logprob"] = logp.gather(1, out["top_idx"])
    return out


# ------------------------------------------------------------------------------ the library


def _own(s):
    import paper_2608_02560_gb300 as precog
    c = s["case"]
    if c["op"] == "delta":
        inputs = precog.delta_inputs(s["q"] if s["y"] is not None else None, s["k"], s["v"], s["g"], s["beta"])
        precog.precog_delta_scan(inputs, s["offsets"], s["T"], bank=s["bank"], idx=s["idx"], layer=c["layer"],
                                 y_out=s["y"], states_out=s["states"])
        return {"y": s["y"], "states": s["states"]}
    if c["op"] == "step":
        inputs = precog.delta_inputs(s["q"], s["k"], s["v"], s["g"], s["beta"])
        precog.precog_delta_step(inputs, s["states"], slots=s["slots"], layer=c["layer"], y_out=s["y"])
        return {"y": s["y"], "states": s["states"]}
    if c["op"] == "qk":
        precog.precog_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], norm=c["norm"], q_weight=s["wq"],
                                   k_weight=s["wk"], eps=1e-6, cos=s["cos"], sin=s["sin"], positions=s["pos"],
                                   interleaved=c["inter"])
        return {"q": s["q_out"], "k": s["k_out"]}
    precog.precog_token_logprobs(s["logits"], s["tokens"], s["logprob"], entropy=s["entropy"], top_idx=s["top_idx"],
                                 top_logprob=s["top_logprob"], temperature=c["temp"])
    out = {"logprob": s["logprob"], "entropy": s["entropy"]}
    if c["k"]:
        out["top_idx"], out["top_logprob"] = s["top_idx"], s["top_logprob"]
    return out


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "delta":
        return _plain_delta(state)
    if op == "step":
        return _plain_step(state)
    if op == "qk":
        return {"q": _plain_qk_one(state["q"], state["wq"], state), "k": _plain_qk_one(state["k"], state["wk"], state)}
    return _plain_logprobs(state)


# ------------------------------------------------------------------------------ 64 bits


def _exact_delta(c, s):
    """Token after token, as the rule is defined; sequences sorted by length, so that each
    token's turn concerns the first of them only."""
    want_y = s["y"] is not None
    order = sorted(range(c["n"]), key=lambda i: -s["lens"][i])
    lens = [s["lens"][i] for i in order]
    if max(lens) > 40000 or sum(lens) * c["hv"] * c["dk"] * c["dv"] > 2e11:
        return None
    perm = torch.tensor(order, device=DEV)
    first = s["offsets"][:-1][perm]
    S = _start_states(s, torch.float64)[perm]                                   # [n, Hv, dv, dk]
    y = torch.zeros((s["T"], c["hv"], c["dv"]), dtype=torch.float64, device=DEV) if want_y else None
    group = torch.arange(c["hv"], device=DEV) // (c["hv"] // c["hk"])
    alive = c["n"]
    for t in range(lens[0]):
        while lens[alive - 1] <= t:
            alive -= 1
        row = first[:alive] + t
        k, v = s["k"][row].double()[:, group], s["v"][row].double()
        H = S[:alive]
        H *= torch.exp(s["g"][row].double())[..., None, None]
        u = s["beta"][row].double()[..., None] * (v - torch.matmul(H, k[..., None])[..., 0])
        H.addcmul_(u[..., None], k[..., None, :])
        if want_y:
            q = s["q"][row].double()[:, group]
            y[row] = c["dk"] ** -0.5 * torch.matmul(H, q[..., None])[..., 0]
    states = torch.zeros((c["n"], c["layers"], c["hv"], c["dv"], c["dk"]), dtype=torch.float64, device=DEV)
    states[perm, c["layer"]] = S
    return {"y": y, "states": states}


def _exact_step(c, s):
    table = s["states"].double()
    group = torch.arange(c["hv"], device=DEV) // (c["hv"] // c["hk"])
    k, q = s["k"].double()[:, group], s["q"].double()[:, group]
    S = table[s["slots"], c["layer"]]
    a = torch.exp(s["g"].double())[..., None]
    b = s["beta"].double()[..., None]
    old = torch.einsum("nhvk,nhk->nhv", S, k)
    S = a[..., None] * (S - b[..., None] * torch.einsum("nhv,nhk->nhvk", old, k))
    S = S + torch.einsum("nhv,nhk->nhvk", b * s["v"].double(), k)
    table[s["slots"], c["layer"]] = S
    return {"y": torch.einsum("nhvk,nhk->nhv", S, q) / math.sqrt(c["dk"]), "states": table}


def _exact_qk_one(x, w, c, s):
    x = x.double()
    n = torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2
    x = x if c["norm"] == "none" else x / torch.sqrt((n if c["norm"] == "l2" else n / c["d"]) + 1e-6)
    x = x if w is None else x * w.double()
    if not c["rot"]:
        return x
    half = torch.arange(c["rot"] // 2, device=DEV)
    at = (2 * half, 2 * half + 1) if c["inter"] else (half, half + c["rot"] // 2)
    z = torch.complex(x[..., at[0]], x[..., at[1]])
    z = z * torch.complex(s["cos"][s["pos"]].double(), s["sin"][s["pos"]].double())[:, None]
    out = x.clone()
    out[..., at[0]], out[..., at[1]] = z.real, z.imag
    return out


def _exact_logprobs(c, s):
    z = s["logits"].double() / c["temp"]
    lse = torch.logsumexp(z, -1, keepdim=True)
    logp = z - lse
    p = torch.exp(logp)
    out = {"logprob": logp[torch.arange(c["rows"], device=DEV), s["tokens"]],
           "entropy": -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(-1)}
    if c["k"]:
        top = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True).indices[:, :c["k"]]
        out["top_idx"], out["top_logprob"] = top, logp.gather(1, top)
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "delta":
        return _exact_delta(c, s)
    if c["op"] == "step":
        return _exact_step(c, s)
    if c["op"] == "qk":
        return {"q": _exact_qk_one(s["q"], s["wq"], c, s), "k": _exact_qk_one(s["k"], s["wk"], c, s)}
    return _exact_logprobs(c, s)


# ------------------------------------------------------------------------------ least work


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "delta":
        T = c["n"] * (c["least"] + c["most"]) / 2
        y = c["y"] != "none"
        size = {"none": 0, "bf16": 2, "f32": 4}
        state = c["n"] * c["hv"] * c["dv"] * c["dk"]
        rows = c["hk"] * c["dk"] * (2 if y else 1) * e + c["hv"] * c["dv"] * (e + size[c["y"]]) + 8 * c["hv"]
        return {"bytes": T * rows + state * (size[c["bank"]] + size[c["out"]]),
                "flops": T * c["hv"] * c["dk"] * c["dv"] * (6 if y else 4)}
    if c["op"] == "step":
        state = c["n"] * c["hv"] * c["dv"] * c["dk"]
        return {"bytes": 8 * state + c["n"] * (2 * c["hk"] * c["dk"] * e + 2 * c["hv"] * c["dv"] * e + 8 * c["hv"]),
                "flops": 6 * state}
    if c["op"] == "qk":
        n = c["tokens"] * (c["hq"] + c["hk"]) * c["d"]
        used = min(c["tokens"], c["positions"])
        return {"bytes": 2 * n * e + (used * c["rot"] * 4 + 8 * c["tokens"] if c["rot"] else 0), "flops": 7 * n}
    n = c["rows"] * c["vocab"]
    return {"bytes": n * e + c["rows"] * (16 + 12 * c["k"]), "flops": 6 * n}
