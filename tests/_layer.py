"""Error bounds of the convolution, the scan's single tokens, the block norm and the adjusted logits, entry by
entry, from how many roundings stand behind each (no method arithmetic beyond the exponentials they need).

A rounding to fp32 is 2^-24 of a value. SiLU of fp32 rows: an exponential within 2 units of 2^-23, a sum and a
quotient, 2^-21 of the value at most. Of 16-bit rows: an exponential within 2 + 1.173 |x| units and a quotient
within 2, (5 + 1.2 |x|) 2^-23. An output in 16 bits is rounded once more, by eps / 2."""
import numpy as np

U = 2.0 ** -24
HALF = {"float32": U, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def name(dtype) -> str:
    return str(dtype).split(".")[-1]


def silu_rel(x, dtype) -> np.ndarray:
    return np.full(np.shape(x), 8 * U) if name(dtype) == "float32" else (5 + 1.2 * np.abs(x)) * 2 * U


def close(got, ref, bound, dtype):
    """got (stored as dtype) within bound of ref besides its own rounding; NaN and infinity in their places."""
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    assert got.shape == ref.shape
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    inf = np.isinf(ref)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(np.sign(got[inf]), np.sign(ref[inf]))
    fine = np.isfinite(ref)
    bound = np.broadcast_to(bound, ref.shape)[fine]
    tiny = 2.0 ** -24 if name(dtype) == "float16" else 1e-30     # fp16 below its normal numbers, and flushed terms
    off = np.abs(got[fine] - ref[fine]) - (bound + HALF[name(dtype)] * (np.abs(ref[fine]) + bound) + tiny)
    assert not off.size or float(off.max()) <= 0.0, (float(off.max()), float(bound.max()))


def conv_bound(x, weight, offsets, bias, act, windows, ref, dtype):
    """K products and a bias added in fp32: K + 1 roundings of the sum of magnitudes; SiLU's slope is below 1.1."""
    import oracle
    K = weight.shape[1]
    mag, _ = oracle.causal_conv(np.abs(x), np.abs(weight), offsets, None if bias is None else np.abs(bias), False,
                                None if windows is None else [np.abs(w) for w in windows])
    if not act:
        return (K + 1) * U * mag
    # |silu(a)| and a differ by less than |a|'s tail: its relative error at |a| <= mag
    return 1.1 * (K + 1) * U * mag + silu_rel(mag, dtype) * np.abs(ref)


def step_bound(x, dt, A, B, C, h0, h, y, skip, gate, dtype):
    """The exponent (two roundings of it), the exponential (2^-22), a product and a sum; complex states turn by
    an angle whose sine and cosine are within 2^-22 and are products of two sums more."""
    import oracle
    z = np.abs(dt[:, :, None] * A.real) if np.iscomplexobj(A) else np.abs(dt[:, :, None] * A)
    decayed = np.exp(np.minimum(dt[:, :, None] * A.real, 700.0)) * np.abs(h0)
    u = np.abs((x * dt)[:, :, None] * B[:, None, :])
    state = decayed * (2 * z + (24 if np.iscomplexobj(A) else 8)) * U + 4 * U * u + 1e-36 * np.abs(h0)
    ch = (np.abs(C)[:, None, :] * np.abs(h.real)).sum(-1)
    out = (np.abs(C)[:, None, :] * state).sum(-1) + 20 * U * ch
    if skip is not None:
        out = out + 3 * U * np.abs(skip * x)
    if gate is not None:
        out = out * np.abs(oracle.silu(gate)) + (silu_rel(gate, dtype) + 2 * U) * np.abs(y)
    return state, out


def _normed(value, err, weight, groups, eps):
    """The root of a sum of n squares, at most 64 roundings in a chain (halved by the root), and two products."""
    T = value.shape[0]
    v, e = value.reshape(T, groups, -1), err.reshape(T, groups, -1)
    root = np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    rel = np.sqrt((e * e).mean(-1, keepdims=True)) / root + 40 * U
    return ((e + rel * np.abs(v)) / root).reshape(value.shape) * np.abs(weight)


def norm_bound(args, dtype, eps=1e-6):
    """Errors of (out, residual_out) of oracle.block_norm(**args)."""
    import oracle
    a = args["x"]
    err = np.zeros_like(a)
    if args.get("skip") is not None:
        more = args["skip"] * args["skip_input"]
        a, err = a + more, 2 * U * (np.abs(a) + np.abs(more))

    def gated(a, err):
        s = oracle.silu(args["gate"])
        return a * s, err * np.abs(s) + (silu_rel(args["gate"], dtype) + 2 * U) * np.abs(a * s)

    first = args.get("gate_first", True)
    if args.get("gate") is not None and first:
        a, err = gated(a, err)
    if args.get("norm", True):
        w = 1.0 if args.get("weight") is None else args["weight"]
        err = _normed(a, err, w, args.get("groups", 1), eps)
        a = oracle.rms(a, eps, args.get("groups", 1)) * w
    if args.get("gate") is not None and not first:
        a, err = gated(a, err)
    if args.get("residual") is None:
        return err, None
    scale = args.get("scale", 1.0)
    h = args["residual"] + scale * a
    err = np.abs(scale) * err + 4 * U * (np.abs(args["residual"]) + np.abs(scale * a))
    w = 1.0 if args.get("out_weight") is None else args["out_weight"]
    return (_normed(h, err, w, 1, eps) if args.get("out_norm") else None), err
