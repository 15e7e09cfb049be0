"""The operators around a selective state space layer and its answers, as timed and compared cases.

Kinds of case (``case["op"]``):

* ``conv``      -- the short causal convolution with SiLU over a ragged batch of sequences, each from
  a retrieved window of inputs (or from none), leaving the window that its next token needs;
* ``conv_step`` -- the same for one token of each sequence of a serving batch, on a table of windows;
* ``scan_step`` -- one token of the diagonal selective scan of each sequence, on a table of fp32
  states (real or complex), with the input's skip and the gate;
* ``norm``      -- the end of a block: skip, gate, RMS norm (of groups), the residual with its scale,
  and the norm that the next block begins with;
* ``adjust``    -- logits before a token is chosen: penalties for repeated tokens, biases, grammar masks.

Shapes: conv x ``[T, D]``, weight ``[D, K]``, windows ``[entries, layers, K - 1, D]`` (oldest input
first); scan x, dt ``[L, n, D]``, B, C ``[L, n, 16]``, A ``[L, D, 16]``, states
``[slots, layers, D, 16]``; norm rows ``[T, D]``; logits ``[R, V]``, masks one bit a token in int32
words ``[masks, ceil(V / 32)]``.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"
N = 16


def listed():
    return [
        # One user's question of 64 tokens behind a retrieved chunk: a call's latency.
        dict(name="conv_question", op="conv", n=1, least=64, most=64, tail=0, dim=2048, k=4, dtype="bf16", bias=True,
             silu=True, entries=16, layers=2, layer=1, pad=0),
        # A server's batch of questions of odd lengths, slices of a wider projection, in a padded buffer.
        dict(name="conv_questions", op="conv", n=96, least=0, most=200, tail=57, dim=2048, k=4, dtype="bf16",
             bias=True, silu=True, entries=64, layers=1, layer=0, pad=2048),
        # Bulk indexing of a ragged corpus from empty windows.
        dict(name="conv_corpus", op="conv", n=256, least=256, most=4096, tail=0, dim=2048, k=4, dtype="bf16",
             bias=True, silu=True, entries=0, layers=1, layer=0, pad=0),
        # One answer token of one user.
        dict(name="conv_step_one", op="conv_step", n=1, slots=4, dim=2048, k=4, dtype="bf16", bias=True, silu=True,
             layers=1, layer=0, pad=2048),
        # One token of each of 256 users' answers, wide channels (x, B and C of a layer together).
        dict(name="conv_step_batch", op="conv_step", n=256, slots=300, dim=8448, k=4, dtype="bf16", bias=True,
             silu=True, layers=1, layer=0, pad=0),
        # One answer token of one user through 24 layers' states of 256 channels.
        dict(name="scan_step_one", op="scan_step", n=1, slots=4, depth=24, dim=256, cplx=False, dtype="bf16",
             skip=True, gate=True, layers=24, layer=0),
        # One token of each of 256 users' answers in a wide layer: the states pass through memory once.
        dict(name="scan_step_batch", op="scan_step", n=256, slots=300, depth=1, dim=4096, cplx=False, dtype="bf16",
             skip=True, gate=True, layers=2, layer=1),
        # One token between two blocks: the residual in fp32 and the next block's norm.
        dict(name="norm_one", op="norm", tokens=1, dim=2048, groups=1, dtype="bf16", res="f32", skip=False,
             gate="none", norm=False, scale="none", out_norm=True, pad=0),
        # A corpus batch inside a block: skip, gate, then the norm of what the scan read out.
        dict(name="norm_gated_corpus", op="norm", tokens=65521, dim=4096, groups=1, dtype="bf16", res="none",
             skip=True, gate="before", norm=True, scale="none", out_norm=False, pad=4096),
        # The same batch between two blocks: norm behind the block, scaled residual, norm before the next.
        dict(name="norm_residual_corpus", op="norm", tokens=65521, dim=2048, groups=1, dtype="bf16", res="f32",
             skip=False, gate="none", norm=True, scale="vector", out_norm=True, pad=0),
        # The next token of one answer of some hundred tokens.
        dict(name="adjust_one", op="adjust", rows=1, vocab=32000, pad=0, dtype="bf16", least=700, most=700,
             prompt=0.5, rep=True, count=True, bias=0, masks=0, allowed=1.0),
        # A decoding batch with long histories, a few biases, and grammars that allow few tokens.
        dict(name="adjust_batch", op="adjust", rows=256, vocab=128001, pad=7, dtype="bf16", least=0, most=4096,
             prompt=0.8, rep=True, count=True, bias=16, masks=40, allowed=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv", "conv", "conv_step", "scan_step", "scan_step", "norm", "norm", "adjust", "adjust"])
    c = dict(op=op)
    if op in ("conv", "conv_step"):
        c.update(dim=8 * _log(rng, 1, 1200), k=rng.choice([2, 3, 4, 4]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 bias=rng.random() < 0.7, silu=rng.random() < 0.8, layers=rng.randint(1, 3),
                 pad=rng.choice([0, 8 * rng.randint(1, 400)]))
        c["layer"] = rng.randrange(c["layers"])
        if op == "conv_step":
            c["n"] = _log(rng, 1, 256)
            c["slots"] = c["n"] + rng.randint(0, 50)
            return c
        c["n"] = _log(rng, 1, 256)
        most = min(_log(rng, 1, 16384), int(4e8 / (c["n"] * (c["dim"] + c["pad"]))))
        c["most"] = max(1, most)
        c.update(least=rng.randint(0, c["most"]), entries=rng.choice([0, rng.randint(1, 2 * c["n"])]),
                 tail=rng.choice([0, 0, rng.randint(1, 100)]))
        return c
    if op == "scan_step":
        c.update(n=_log(rng, 1, 256), depth=rng.choice([1, 1, rng.randint(1, 24)]), dim=8 * _log(rng, 1, 600),
                 cplx=rng.random() < 0.25, dtype=rng.choice(["bf16", "bf16", "f32"]), skip=rng.random() < 0.6,
                 gate=rng.random() < 0.6)
        c["depth"] = max(1, min(c["depth"], int(2e6 / (c["n"] * c["dim"]))))
        c["layers"] = c["depth"] + rng.randint(0, 2)
        c["layer"] = rng.randint(0, c["layers"] - c["depth"])
        c["slots"] = c["n"] + rng.randint(0, 50)
        return c
    if op == "norm":
        res = rng.choice(["none", "f32", "f32", "bf16"])
        c.update(dim=8 * _log(rng, 1, 1024), res=res, dtype="bf16" if res == "bf16" else rng.choice(["bf16", "f32"]),
                 skip=rng.random() < 0.4, gate=rng.choice(["none", "before", "after"]), norm=rng.random() < 0.7,
                 scale="none" if res == "none" else rng.choice(["none", "scalar", "vector"]),
                 out_norm=res != "none" and rng.random() < 0.8, pad=rng.choice([0, 8 * rng.randint(1, 400)]))
        c["tokens"] = max(1, min(_log(rng, 1, 65536), int(1e8 / (c["dim"] + c["pad"]))))
        c["groups"] = 1
        if c["norm"] and not c["out_norm"] and rng.random() < 0.5:
            c["groups"] = rng.choice([g for g in (1, 2, 4, 8, 16, 32, 64) if c["dim"] % (8 * g) == 0])
        return c
    vocab = _log(rng, 100, 152000)
    c.update(vocab=vocab, rows=max(1, min(_log(rng, 1, 512), int(3.0e7 / vocab))), pad=rng.randint(0, 9),
             dtype=rng.choice(["bf16", "f32", "f16"]), most=_log(rng, 1, 8192), prompt=rng.choice([0.0, 0.5, 0.9]),
             rep=rng.random() < 0.7, count=rng.random() < 0.7, bias=rng.choice([0, rng.randint(1, 60)]),
             masks=rng.choice([0, rng.randint(1, 64)]), allowed=rng.choice([0.02, 0.5, 0.99]))
    c["least"] = rng.randint(0, c["most"])
    return c


def _lens(case, seed):
    """The case's lengths, in an order of the seed's (so that every seed has as many tokens)."""
    r = random.Random(29)
    count = case["n"] if case["op"] == "conv" else case["rows"]
    lens = [r.randint(case["least"], case["most"]) for _ in range(count)]
    if case["op"] == "conv" and sum(lens) == 0:
        lens[0] = 1
    random.Random(int(seed)).shuffle(lens)
    return lens


def _offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return torch.tensor(off, dtype=torch.int64, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1013 + 29)
    rand = lambda *shape: torch.randn(shape, device=DEV, generator=gen)  # noqa: E731
    c, dt = dict(case), DTYPES[case["dtype"]]
    s = {"case": c}
    if c["op"] in ("conv", "conv_step"):
        D, K = c["dim"], c["k"]
        if c["op"] == "conv":
            s["lens"] = _lens(c, seed)
            s["offsets"] = _offsets(s["lens"])
            T = sum(s["lens"]) + c["tail"]
            s["bank"] = s["idx"] = None
            if c["entries"]:
                s["bank"] = rand(c["entries"], c["layers"], K - 1, D).to(dt)
                # retrieved rows; -1 where nothing was comparable
                s["idx"] = torch.randint(-1, c["entries"], (c["n"],), device=DEV, generator=gen)
            s["windows"] = torch.zeros((c["n"], c["layers"], K - 1, D), dtype=dt, device=DEV)
        else:
            T = c["n"]
            s["windows"] = rand(c["slots"], c["layers"], K - 1, D).to(dt)
            s["slots"] = torch.randperm(c["slots"], device=DEV, generator=gen)[:T].contiguous()
        wide = torch.empty((T, D + c["pad"]), dtype=dt, device=DEV)
        for at in range(0, T, 1 << 16):
            wide[at:at + (1 << 16)] = rand(min(1 << 16, T - at), D + c["pad"])
        s["x"] = wide[:, :D]
        s["weight"] = 0.5 * rand(D, K)
        s["bias"] = 0.3 * rand(D) if c["bias"] else None
        s["y"] = torch.zeros((T, D), dtype=dt, device=DEV)
        return s
    if c["op"] == "scan_step":
        L, n, D = c["depth"], c["n"], c["dim"]
        s["x"] = rand(L, n, D).to(dt)
        s["dt"] = torch.nn.functional.softplus(rand(L, n, D) - 2.0).to(dt)
        s["B"], s["C"] = ((0.25 * rand(L, n, N)).to(dt) for _ in range(2))
        rate = torch.arange(1, N + 1, device=DEV) * torch.exp(0.3 * rand(L, D, 1))
        s["A"] = -rate
        if c["cplx"]:
            turn = math.pi * torch.arange(N, device=DEV, dtype=torch.float32)
            s["A"] = torch.complex(-rate, turn.expand(L, D, N).contiguous())
        s["states"] = 0.3 * rand(c["slots"], c["layers"], D, N, *((2,) if c["cplx"] else ()))
        if c["cplx"]:
            s["states"] = torch.view_as_complex(s["states"])
        s["slots"] = torch.randperm(c["slots"], device=DEV, generator=gen)[:n].contiguous()
        s["skip"] = rand(L, D) if c["skip"] else None
        s["gate"] = rand(L, n, D).to(dt) if c["gate"] else None
        s["y"] = torch.zeros((L, n, D), dtype=dt, device=DEV)
        return s
    if c["op"] == "norm":
        T, D = c["tokens"], c["dim"]
        s["x"] = rand(T, D).to(dt)
        s["u"] = rand(T, D).to(dt) if c["skip"] else None
        s["skip"] = rand(D) if c["skip"] else None
        s["gate"] = rand(T, D + c["pad"]).to(dt)[:, c["pad"]:] if c["gate"] != "none" else None
        s["weight"] = 1.0 + 0.2 * rand(D) if c["norm"] else None
        s["out_weight"] = 1.0 + 0.2 * rand(D) if c["out_norm"] else None
        s["scale"] = {"none": 1.0, "scalar": 0.7, "vector": None}[c["scale"]]
        if c["scale"] == "vector":
            s["scale"] = 0.3 * rand(D)
        s["residual"] = s["residual_out"] = s["out"] = None
        if c["res"] != "none":
            s["residual"] = (3.0 * rand(T, D)).to(DTYPES[c["res"]])
            s["residual_out"] = torch.zeros_like(s["residual"])
        if c["res"] == "none" or c["out_norm"]:
            s["out"] = torch.zeros((T, D), dtype=dt, device=DEV)
        return s
    R, V = c["rows"], c["vocab"]
    s["lens"] = _lens(c, seed)
    s["logits"] = (2.5 * rand(R, V + c["pad"])).to(dt)[:, :V]
    s["out"] = torch.zeros((R, V), dtype=dt, device=DEV)
    s["offsets"] = _offsets(s["lens"])
    # tokens as texts have them: few of them often, most of them rarely
    u = torch.rand(sum(s["lens"]), device=DEV, generator=gen, dtype=torch.float64)
    s["history"] = torch.exp(u * math.log(V)).long().clamp(max=V) - 1
    s["count_from"] = (c["prompt"] * (s["offsets"][1:] - s["offsets"][:-1])).long()
    s["rep"] = 1.0 + 0.5 * torch.rand(R, device=DEV, generator=gen) if c["rep"] else None
    s["freq"] = 0.3 * torch.rand(R, device=DEV, generator=gen) if c["count"] else None
    s["pres"] = 0.3 * torch.rand(R, device=DEV, generator=gen) if c["count"] else None
    s["bias_idx"] = s["bias_val"] = s["bias_offsets"] = s["mask"] = s["mask_rows"] = None
    b = min(c["bias"], V)
    if b:
        s["bias_idx"] = torch.rand((R, V), device=DEV, generator=gen).topk(b, dim=1).indices.reshape(-1).contiguous()
        s["bias_val"] = 2.0 * rand(R * b)
        s["bias_offsets"] = b * torch.arange(R + 1, device=DEV)
    if c["masks"]:
        bits = torch.rand((c["masks"], (V + 31) // 32, 32), device=DEV, generator=gen) < c["allowed"]
        words = (bits.long() << torch.arange(32, device=DEV)).sum(-1)
        s["mask"] = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
        # -1: a request without a grammar
        s["mask_rows"] = torch.randint(-1, c["masks"], (R,), device=DEV, generator=gen)
    return s


# ------------------------------------------------------------------------------ plain forms


def _silu(z):
    return z / (1.0 + torch.exp(-z))


def _plain_conv(s):
    c, K = s["case"], s["case"]["k"]
    first, last = s["offsets"][:-1], s["offsets"][1:]
    lens = last - first
    T = sum(s["lens"])
    x = s["x"][:T]
    if s["bank"] is None:
        before = torch.zeros((c["n"], K - 1, c["dim"]), dtype=x.dtype, device=DEV)
    else:
        before = s["bank"][s["idx"].clamp(min=0), c["layer"]] * (s["idx"] >= 0).to(x.dtype)[:, None, None]
    acc = x.float() * s["weight"][:, K - 1]
    rows = torch.empty((T + 1, c["dim"]), device=DEV)           # the last row: nobody's
    for back in range(1, K):
        rows[:min(back, T)] = 0.0
        rows[back:T] = x[:max(T - back, 0)]
        place = torch.arange(back, device=DEV)                  # the first tokens' inputs are the window's
        to = torch.where(place < lens[:, None], first[:, None] + place, T)
        rows[to] = before[:, K - 1 - back:].float()
        acc += rows[:T] * s["weight"][:, K - 1 - back]
    if s["bias"] is not None:
        acc += s["bias"]
    s["y"][:T] = (_silu(acc) if c["silu"] else acc).to(s["y"].dtype)
    j = torch.arange(K - 1, device=DEV)
    src = lens[:, None] - (K - 1) + j                           # place of the window's j-th input
    old = before.gather(1, (src + K - 1).clamp(max=K - 2)[..., None].expand(-1, -1, c["dim"]))
    new = x[(first[:, None] + src).clamp(min=0, max=T - 1)]
    s["windows"][:, c["layer"]] = torch.where((src < 0)[..., None], old, new)
    return {"y": s["y"], "windows": s["windows"]}


def _plain_conv_step(s):
    c = s["case"]
    win = torch.cat((s["windows"][s["slots"], c["layer"]], s["x"][:, None]), 1)          # [n, K, D]
    acc = (win.float() * s["weight"].t()).sum(1)
    if s["bias"] is not None:
        acc = acc + s["bias"]
    s["windows"][s["slots"], c["layer"]] = win[:, 1:]
    return {"y": (_silu(acc) if c["silu"] else acc).to(s["y"].dtype), "windows": s["windows"]}


def _plain_scan_step(s):
    c = s["case"]
    at = slice(c["layer"], c["layer"] + c["depth"])
    x, dt, B, C = (s[k].float().transpose(0, 1) for k in ("x", "dt", "B", "C"))          # [n, L, ...]
    h = s["states"][s["slots"], at]
    h = torch.exp(dt[..., None] * s["A"]) * h + (x * dt)[..., None] * B[:, :, None, :]
    s["states"][s["slots"], at] = h
    y = ((h.real if c["cplx"] else h) * C[:, :, None, :]).sum(-1)
    if s["skip"] is not None:
        y = y + s["skip"] * x
    if s["gate"] is not None:
        y = y * _silu(s["gate"].float().transpose(0, 1))
    states = torch.view_as_real(s["states"]) if c["cplx"] else s["states"]
    return {"y": y.transpose(0, 1).to(s["y"].dtype).contiguous(), "states": states}


def _rms(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def _plain_norm(s):
    c = s["case"]
    T, D, G = c["tokens"], c["dim"], c["groups"]
    a = s["x"].float()
    if c["skip"]:
        a = a + s["skip"] * s["u"].float()
    if c["gate"] == "before":
        a = a * _silu(s["gate"].float())
    if c["norm"]:
        a = _rms(a.view(T, G, D // G), s["weight"].view(G, D // G)).view(T, D)
    if c["gate"] == "after":
        a = a * _silu(s["gate"].float())
    if c["res"] == "none":
        return {"out": a.to(s["x"].dtype), "residual": None}
    h = s["residual"].float() + s["scale"] * a
    out = _rms(h, s["out_weight"]).to(s["x"].dtype) if c["out_norm"] else None
    return {"out": out, "residual": h.to(s["residual"].dtype)}


def _plain_adjust(s):
    c = s["case"]
    R, V = c["rows"], c["vocab"]
    z = s["logits"].float()
    lens = s["offsets"][1:] - s["offsets"][:-1]
    total = sum(s["lens"])
    row = torch.arange(R, device=DEV).repeat_interleave(lens, output_size=total)
    one = torch.ones(total, dtype=torch.int32, device=DEV)
    if c["rep"]:
        seen = torch.zeros((R, V), dtype=torch.int32, device=DEV).index_put_((row, s["history"]), one, accumulate=True)
        p = s["rep"][:, None]
        z = torch.where(seen > 0, torch.where(z > 0, z / p, z * p), z)
    if c["count"]:
        late = torch.arange(total, device=DEV) - s["offsets"][:-1][row] >= s["count_from"][row]
        count = torch.zeros((R, V), dtype=torch.int32, device=DEV).index_put_((row, s["history"]), one * late,
                                                                             accumulate=True)
        z = torch.where(count > 0, z - s["freq"][:, None] * count - s["pres"][:, None], z)
    if s["bias_idx"] is not None:
        of = torch.arange(R, device=DEV).repeat_interleave(s["bias_idx"].numel() // R)
        z[of, s["bias_idx"]] += s["bias_val"]
    if s["mask"] is not None:
        i = torch.arange(V, device=DEV)
        banned = ((s["mask"][:, i >> 5] >> (i & 31)) & 1) == 0
        z = z.masked_fill(banned[s["mask_rows"].clamp(min=0)] & (s["mask_rows"] >= 0)[:, None], -math.inf)
    return {"logits": z.to(s["out"].dtype)}


# ------------------------------------------------------------------------------ the library


def _own(s):
    import paper_2608_02560_gb300 as precog
    c = s["case"]
    if c["op"] == "conv":
        precog.precog_causal_conv(s["x"], s["weight"], s["offsets"], bias=s["bias"], silu=c["silu"], bank=s["bank"],
                                  idx=s["idx"], layer=c["layer"], windows_out=s["windows"], y_out=s["y"])
        return {"y": s["y"], "windows": s["windows"]}
    if c["op"] == "conv_step":
        precog.precog_conv_step(s["x"], s["weight"], s["windows"], slots=s["slots"], bias=s["bias"], silu=c["silu"],
                                layer=c["layer"], y_out=s["y"])
        return {"y": s["y"], "windows": s["windows"]}
    if c["op"] == "scan_step":
        kind = precog.PRECOG_A_COMPLEX if c["cplx"] else precog.PRECOG_A_GENERAL
        inputs = precog.scan_inputs(s["x"], s["dt"], s["B"], s["A"], s["C"], a_kind=kind)
        precog.precog_scan_step(inputs, s["states"], slots=s["slots"], layer0=c["layer"], skip=s["skip"],
                                gate=s["gate"], y_out=s["y"])
        return {"y": s["y"], "states": torch.view_as_real(s["states"]) if c["cplx"] else s["states"]}
    if c["op"] == "norm":
        precog.precog_block_norm(s["x"], out=s["out"], skip=s["skip"], skip_input=s["u"], gate=s["gate"],
                                 gate_first=c["gate"] == "before", weight=s["weight"], groups=c["groups"],
                                 residual=s["residual"], scale=s["scale"], residual_out=s["residual_out"],
                                 out_weight=s["out_weight"], eps=1e-6)
        return {"out": s["out"], "residual": s["residual_out"]}
    precog.precog_adjust_logits(s["logits"], s["out"], history=s["history"] if c["rep"] or c["count"] else None,
                                history_offsets=s["offsets"], count_from=s["count_from"], repetition=s["rep"],
                                frequency=s["freq"], presence=s["pres"], bias_idx=s["bias_idx"],
                                bias=s["bias_val"], bias_offsets=s["bias_offsets"], mask=s["mask"],
                                mask_rows=s["mask_rows"])
    return {"logits": s["out"]}


def run(state):
    if own:
        return _own(state)
    return {"conv": _plain_conv, "conv_step": _plain_conv_step, "scan_step": _plain_scan_step, "norm": _plain_norm,
            "adjust": _plain_adjust}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------ 64 bits


def _act64(c, acc):
    return acc * torch.sigmoid(acc) if c["silu"] else acc


def _exact_conv(c, s):
    """Sequence after sequence: its window and its tokens one behind the other, unfolded."""
    K = c["k"]
    y = s["y"].double()
    windows = s["windows"].double()
    rows = s["idx"].tolist() if s["idx"] is not None else [-1] * c["n"]
    at = 0
    for i, n in enumerate(s["lens"]):
        old = s["bank"][rows[i], c["layer"]].double() if rows[i] >= 0 else torch.zeros_like(windows[0, 0])
        whole = torch.cat((old, s["x"][at:at + n].double()))
        if n:
            acc = torch.einsum("tdk,dk->td", whole.unfold(0, K, 1), s["weight"].double())
            y[at:at + n] = _act64(c, acc if s["bias"] is None else acc + s["bias"].double())
        windows[i, c["layer"]] = whole[n:]
        at += n
    return {"y": y, "windows": windows}


def _exact_conv_step(c, s):
    windows = s["windows"].double()
    y = torch.empty(s["y"].shape, dtype=torch.float64, device=DEV)
    for i, slot in enumerate(s["slots"].tolist()):
        whole = torch.cat((windows[slot, c["layer"]], s["x"][i:i + 1].double()))
        acc = torch.einsum("kd,dk->d", whole, s["weight"].double())
        y[i] = _act64(c, acc if s["bias"] is None else acc + s["bias"].double())
        windows[slot, c["layer"]] = whole[1:]
    return {"y": y, "windows": windows}


def _exact_scan_step(c, s):
    wide = torch.complex128 if c["cplx"] else torch.float64
    states = s["states"].to(wide)
    y = torch.empty(s["y"].shape, dtype=torch.float64, device=DEV)
    for layer in range(c["depth"]):
        h = states[s["slots"], c["layer"] + layer]
        x, dt = s["x"][layer].double(), s["dt"][layer].double()
        h = h * torch.exp(torch.einsum("nd,dk->ndk", dt.to(wide), s["A"][layer].to(wide)))
        h = h + torch.einsum("nd,nk->ndk", x * dt, s["B"][layer].double())
        states[s["slots"], c["layer"] + layer] = h
        y[layer] = torch.einsum("ndk,nk->nd", h.real if c["cplx"] else h, s["C"][layer].double())
        if s["skip"] is not None:
            y[layer] += s["skip"][layer].double() * x
        if s["gate"] is not None:
            z = s["gate"][layer].double()
            y[layer] *= z * torch.sigmoid(z)
    return {"y": y, "states": torch.view_as_real(states) if c["cplx"] else states}


def _exact_norm(c, s):
    def unit(v, parts):
        v = v.reshape(c["tokens"], parts, -1)
        norm2 = torch.linalg.vector_norm(v, dim=-1, keepdim=True) ** 2
        return (v / torch.sqrt(norm2 / v.shape[-1] + 1e-6)).reshape(c["tokens"], -1)

    a = s["x"].double()
    gate = None if s["gate"] is None else s["gate"].double() * torch.sigmoid(s["gate"].double())
    if c["skip"]:
        a = torch.addcmul(a, s["skip"].double(), s["u"].double())
    if c["gate"] == "before":
        a = a * gate
    if c["norm"]:
        a = unit(a, c["groups"]) * s["weight"].double()
    if c["gate"] == "after":
        a = a * gate
    if c["res"] == "none":
        return {"out": a, "residual": None}
    scale = s["scale"].double() if c["scale"] == "vector" else float(s["scale"])
    h = a * scale + s["residual"].double()
    return {"out": unit(h, 1) * s["out_weight"].double() if c["out_norm"] else None, "residual": h}


def _exact_adjust(c, s):
    V = c["vocab"]
    out = s["logits"].double()
    off = s["offsets"].tolist()
    start = s["count_from"].tolist()
    masks = s["mask_rows"].tolist() if s["mask"] is not None else [-1] * c["rows"]
    for r in range(c["rows"]):
        text = s["history"][off[r]:off[r + 1]]
        if c["rep"]:
            there, p = torch.unique(text), s["rep"][r].double()
            v = out[r, there]
            out[r, there] = torch.where(v > 0, v / p, v * p)
        if c["count"]:
            times = torch.bincount(text[start[r]:], minlength=V).double()
            out[r] -= s["freq"][r].double() * times + s["pres"][r].double() * (times > 0)
        if s["bias_idx"] is not None:
            a, b = s["bias_offsets"][r].item(), s["bias_offsets"][r + 1].item()
            out[r, s["bias_idx"][a:b]] += s["bias_val"][a:b].double()
        if masks[r] >= 0:
            words = s["mask"][masks[r]].long() & 0xFFFFFFFF
            allowed = ((words[:, None] >> torch.arange(32, device=DEV)) & 1).reshape(-1)[:V].bool()
            out[r, ~allowed] = -math.inf
    return {"logits": out}


def exact(case, seed):
    s, c = prepare(case, seed), case
    return {"conv": _exact_conv, "conv_step": _exact_conv_step, "scan_step": _exact_scan_step, "norm": _exact_norm,
            "adjust": _exact_adjust}[c["op"]](c, s)


# ------------------------------------------------------------------------------ least work


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "conv":
        T, D = sum(_lens(c, 0)), c["dim"]
        window = c["n"] * (c["k"] - 1) * D * e
        return {"bytes": 2 * T * D * e + window * (2 if c["entries"] else 1) + 4 * D * (c["k"] + c["bias"]),
                "flops": T * D * (2 * c["k"] + (4 if c["silu"] else 0))}
    if c["op"] == "conv_step":
        n = c["n"] * c["dim"]
        return {"bytes": n * e * (2 + 2 * (c["k"] - 1)) + 4 * c["dim"] * (c["k"] + c["bias"]),
                "flops": n * (2 * c["k"] + (4 if c["silu"] else 0))}
    if c["op"] == "scan_step":
        n, parts = c["n"] * c["depth"] * c["dim"], 2 if c["cplx"] else 1
        weights = 4 * c["depth"] * c["dim"] * (N * parts + c["skip"])
        return {"bytes": n * (N * parts * 8 + e * (3 + c["gate"])) + 2 * c["n"] * c["depth"] * N * e + weights,
                "flops": n * N * parts * 7}
    if c["op"] == "norm":
        n = c["tokens"] * c["dim"]
        r = {"none": 0, "f32": 4, "bf16": 2}[c["res"]]
        rows = e * (1 + c["skip"] + (c["gate"] != "none") + (c["res"] == "none" or c["out_norm"])) + 2 * r
        vectors = c["skip"] + c["norm"] + c["out_norm"] + (c["scale"] == "vector")
        return {"bytes": n * rows + 4 * c["dim"] * vectors, "flops": n * 12}
    n = c["rows"] * c["vocab"]
    history = sum(_lens(c, 0)) if c["rep"] or c["count"] else 0
    used = min(c["masks"], c["rows"]) * ((c["vocab"] + 31) // 32) * 4
    return {"bytes": 2 * n * e + 8 * history + 12 * c["rows"] * c["bias"] + used, "flops": 3 * n}
