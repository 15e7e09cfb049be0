"""The gated delta rule against the fp64 recurrence: scans (corpus chunks, injected states,
readout) and single tokens, at the sizes, strides and gates where they can go wrong.

Tolerances, max |gpu - ref| / max |ref| of one output:
* fp32 inputs: TOL_F32 (the suite's; a token adds a few roundings of 2^-24 to a state that
  remembers at most some hundreds of tokens).
* bf16 inputs: TOL_PAIR. Long sequences run in chunks whose intermediate operands are pairs of
  bf16 numbers, each within 2^-17 of its value; five products follow one another in a chunk, and
  the correction's inverse may enlarge an error some fourfold: 5 * 4 * 2^-17 = 1.5e-4.
A bf16 output may differ by its own rounding besides (rel_err_stored)."""
import numpy as np
import pytest

import oracle
from tests._util import TOL_F32, rel_err, rel_err_stored, to_np

pytestmark = pytest.mark.gpu

TOL_PAIR = 1.5e-4


def _tensors(lens, hk, hv, dk, dv, dtype, dev, seed, rate=1.0, strided=False):
    import torch
    gen = torch.Generator(device=dev).manual_seed(seed)
    T = sum(lens)
    rn = lambda *s: torch.randn(s, device=dev, generator=gen)  # noqa: E731
    if strided:
        wide = rn(T, hk * dk * 2 + hv * dv + 16).to(dtype)
        q, k = wide[:, :hk * dk].view(T, hk, dk), wide[:, hk * dk:2 * hk * dk].view(T, hk, dk)
        q /= q.float().norm(dim=-1, keepdim=True).to(dtype)
        k /= k.float().norm(dim=-1, keepdim=True).to(dtype)
        v = wide[:, 2 * hk * dk:2 * hk * dk + hv * dv].view(T, hv, dv)
    else:
        q, k = (torch.nn.functional.normalize(rn(T, hk, dk), dim=-1).to(dtype) for _ in range(2))
        v = rn(T, hv, dv).to(dtype)
    g = -rate * torch.nn.functional.softplus(rn(T, hv) - 2)
    beta = torch.sigmoid(rn(T, hv))
    off = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int64, device=dev)
    return q, k, v, g, beta, off


def _ref(q, k, v, g, beta, off, S0=None):
    return oracle.delta_scan(None if q is None else to_np(q), to_np(k), to_np(v), to_np(g), to_np(beta),
                             off.cpu().numpy(), scale=k.shape[-1] ** -0.5, S0=S0)


def _check(got, ref, tol):
    import torch
    err = rel_err_stored(to_np(got), ref) if got.dtype == torch.bfloat16 else rel_err(to_np(got), ref)
    assert err < tol, err


CASES = [
    # lens, hk, hv, dk, dv, bank, state, y
    ([1], 1, 1, 8, 8, None, "float32", True),
    ([64], 2, 4, 128, 128, "bfloat16", "float32", True),
    ([65, 0, 63, 1, 128, 17], 2, 2, 128, 128, "float32", "bfloat16", True),
    ([200, 3, 129], 1, 3, 64, 64, None, "float32", True),
    ([77, 190], 2, 4, 40, 24, "bfloat16", "float32", True),
    ([300], 1, 2, 128, 200, "float32", "float32", True),
    ([130, 70, 5], 2, 6, 104, 8, None, "bfloat16", False),
    ([257, 64], 3, 3, 72, 136, "bfloat16", "float32", False),
    ([0, 0], 1, 2, 16, 16, "float32", "float32", True),
]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lens,hk,hv,dk,dv,bank,state,want_y", CASES)
def test_scan_matches_the_recurrence(cuda_device, dtype, lens, hk, hv, dk, dv, bank, state, want_y):
    import torch
    import paper_2608_02560_gb300 as pg
    dt, n, L, layer = getattr(torch, dtype), len(lens), 2, 1
    tol = TOL_F32 if dtype == "float32" else TOL_PAIR
    q, k, v, g, beta, off = _tensors(lens, hk, hv, dk, dv, dt, cuda_device, 1 + sum(lens))
    T = int(off[-1])
    b = idx = S0 = None
    if bank:
        gen = torch.Generator(device=cuda_device).manual_seed(5)
        b = torch.randn((n + 2, L, hv, dv, dk), device=cuda_device, generator=gen).to(getattr(torch, bank))
        idx = torch.tensor([(3 * c) % (n + 3) - 1 for c in range(n)], dtype=torch.int64, device=cuda_device)
        S0 = np.stack([to_np(b[i, layer]) if i >= 0 else np.zeros((hv, dv, dk)) for i in idx.tolist()])
    states = torch.full((n, L, hv, dv, dk), 7.0, dtype=getattr(torch, state), device=cuda_device)
    y = torch.full((T, hv, dv), float("nan"), dtype=dt, device=cuda_device) if want_y else None
    pg.precog_delta_scan(pg.delta_inputs(q if want_y else None, k, v, g, beta), off, T, bank=b, idx=idx, layer=layer,
                         states_out=states, y_out=y)
    assert pg.precog_device_status()[0] == 0
    ref_S, ref_y = _ref(q if want_y else None, k, v, g, beta, off, S0)
    assert bool((states[:, 0] == 7.0).all())                   # the other layer is untouched
    _check(states[:, layer], ref_S, tol)
    if want_y and T:
        _check(y, ref_y, tol)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strided_rows_rows_outside_and_bad_offsets(cuda_device, dtype):
    """Slices of one projection; rows before, between and after the sequences hold NaN and
    infinity, which no sequence may see and whose y rows stay untouched."""
    import torch
    import paper_2608_02560_gb300 as pg
    dt = getattr(torch, dtype)
    q, k, v, g, beta, _ = _tensors([400], 2, 4, 64, 72, dt, cuda_device, 9, strided=True)
    begins, ends = [5, 100, 230], [90, 229, 391]
    offs = torch.tensor([5, 90], dtype=torch.int64, device=cuda_device), torch.tensor([100, 229], dtype=torch.int64, device=cuda_device)
    inside = torch.zeros(400, dtype=torch.bool, device=cuda_device)
    for a, b in zip(begins[:2], ends[:2]):
        inside[a:b] = True
    for i, x in enumerate((q, k, v, g, beta)):
        x[~inside] = float("nan") if i % 2 else float("inf")
    for off in offs:
        y = torch.full((400, 4, 72), 3.0, dtype=dt, device=cuda_device)
        s = torch.zeros((1, 1, 4, 72, 64), device=cuda_device)
        pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, 400, states_out=s, y_out=y)
        a, b = off.tolist()
        ref_S, ref_y = _ref(q[a:b], k[a:b], v[a:b], g[a:b], beta[a:b], off - a)
        tol = TOL_F32 if dtype == "float32" else TOL_PAIR
        _check(s[:, 0], ref_S, tol)
        _check(y[a:b], ref_y, tol)
        assert bool((y[:a] == 3.0).all()) and bool((y[b:] == 3.0).all())
    assert pg.precog_device_status()[0] == 0
    # decreasing offsets and offsets beyond T_tot: those sequences are skipped and flagged
    off = torch.tensor([5, 90, 60, 401], dtype=torch.int64, device=cuda_device)
    s = torch.full((3, 1, 4, 72, 64), 7.0, device=cuda_device)
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, 400, states_out=s)
    st, bits = pg.precog_device_status()
    assert st == 5 and bits == pg.PRECOG_DEV_BAD_OFFSETS
    assert bool((s[1:] == 7.0).all()) and bool((s[0] != 7.0).any())


@pytest.mark.parametrize("dtype,n", [("float32", 150), ("bfloat16", 150), ("bfloat16", 3)])
@pytest.mark.parametrize("gates", ["reset", "strong", "none", "growing", "beta0", "beta2"])
def test_gates(cuda_device, dtype, n, gates):
    """Decays of 0 (g = -inf), decays far below fp32 within a chunk, none at all, growth, and the
    ends of beta's range."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, off = _tensors([n], 1, 2, 128, 64, getattr(torch, dtype), cuda_device, 21)
    if gates == "reset":
        g[n // 2] = float("-inf")
        g[n // 3, 0] = -1e30
    elif gates == "strong":
        g *= 60.0
    elif gates == "none":
        g.zero_()
    elif gates == "growing":
        g.fill_(0.05)
    elif gates == "beta0":
        beta.zero_()
    else:
        beta.fill_(2.0)
    S0 = torch.randn((1, 1, 2, 64, 128), device=cuda_device)
    s = torch.empty((1, 1, 2, 64, 128), device=cuda_device)
    y = torch.empty((n, 2, 64), device=cuda_device)
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, n, bank=S0, states_out=s, y_out=y)
    ref_S, ref_y = _ref(q, k, v, g, beta, off, to_np(S0[:, 0]))
    tol = TOL_F32 if dtype == "float32" else TOL_PAIR
    if gates in ("growing", "beta2"):
        tol *= 4      # (|1 - beta k.k| reaches 1, or the state grows e^7.5-fold: errors are kept)
    _check(s[:, 0], ref_S, tol)
    _check(y, ref_y, tol)
    assert pg.precog_device_status()[0] == 0


def test_scan_of_two_parts_equals_the_whole(cuda_device):
    """Theorem 1's form: the state of a chunk, injected, continues as if the chunk had been read."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, off = _tensors([500], 2, 4, 128, 128, torch.bfloat16, cuda_device, 31, rate=0.05)
    whole, part, rest = (torch.empty((1, 1, 4, 128, 128), device=cuda_device) for _ in range(3))
    y, y2 = (torch.zeros((500, 4, 128), device=cuda_device) for _ in range(2))
    inputs = pg.delta_inputs(q, k, v, g, beta)
    pg.precog_delta_scan(inputs, off, 500, states_out=whole, y_out=y)
    cut = torch.tensor([0, 333], dtype=torch.int64, device=cuda_device)
    pg.precog_delta_scan(inputs, cut, 500, states_out=part, y_out=y2)
    cut = torch.tensor([333, 500], dtype=torch.int64, device=cuda_device)
    pg.precog_delta_scan(inputs, cut, 500, bank=part, states_out=rest, y_out=y2)
    assert rel_err(to_np(rest), to_np(whole)) < TOL_PAIR and rel_err(to_np(y2), to_np(y)) < TOL_PAIR


def test_bad_rows_of_the_bank_and_calls_that_repeat(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, off = _tensors([70, 70, 70], 1, 2, 128, 128, torch.bfloat16, cuda_device, 41)
    bank = torch.randn((2, 1, 2, 128, 128), device=cuda_device)
    inputs = pg.delta_inputs(q, k, v, g, beta)
    out = []
    for idx in ([0, 2, -2], [0, -1, -1], [0, -1, -1]):
        s = torch.empty((3, 1, 2, 128, 128), device=cuda_device)
        pg.precog_delta_scan(inputs, off, 210, bank=bank, idx=torch.tensor(idx, device=cuda_device), states_out=s)
        st, bits = pg.precog_device_status()
        assert (st, bits) == ((5, pg.PRECOG_DEV_BAD_INDEX) if idx[1] == 2 else (0, 0))
        out.append(s)
    assert torch.equal(out[0], out[1]) and torch.equal(out[1], out[2])


@pytest.mark.parametrize("T,heads", [(5000, 1), (3001, 2)])
def test_long_sequences(cuda_device, T, heads):
    """Long axes with little to run at once, and the same rows inside a larger batch."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, off = _tensors([T], heads, heads, 64, 64, torch.bfloat16, cuda_device, 51, rate=0.02)
    S0 = torch.randn((1, 1, heads, 64, 64), device=cuda_device)
    s = torch.empty_like(S0)
    y = torch.empty((T, heads, 64), device=cuda_device)
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, T, bank=S0, states_out=s, y_out=y)
    ref_S, ref_y = _ref(q, k, v, g, beta, off, to_np(S0[:, 0]))
    _check(s[:, 0], ref_S, TOL_PAIR)
    _check(y, ref_y, TOL_PAIR)
    assert pg.precog_device_status()[0] == 0


@pytest.mark.parametrize("n,hv,dk,dv,most,y_dtype", [
    (200, 2, 64, 64, 200, "bfloat16"), (170, 1, 128, 136, 130, "float32"), (400, 1, 40, 24, 70, None),
    (160, 1, 128, 128, 1, "bfloat16")])
def test_many_short_sequences(cuda_device, n, hv, dk, dv, most, y_dtype):
    """More items than SMs, of a few chunks each (empty ones among them), and two calls of them: in the
    second one sequence has bad offsets and another a row of the bank that does not exist."""
    import torch
    import paper_2608_02560_gb300 as pg
    r = np.random.default_rng(n)
    lens = [int(x) for x in r.integers(0, most + 1, n)]
    lens[0] = max(most, 9 * n - sum(lens))            # (one of them longer than the rest together)
    q, k, v, g, beta, off = _tensors(lens, 1, hv, dk, dv, torch.bfloat16, cuda_device, n)
    T = sum(lens)
    bank = torch.randn((5, 1, hv, dv, dk), device=cuda_device)
    rows = [int(x) for x in r.integers(-1, 5, n)]
    idx = torch.tensor(rows, device=cuda_device)
    S0 = np.stack([to_np(bank[i, 0]) if i >= 0 else np.zeros((hv, dv, dk)) for i in rows])
    states = torch.full((n, 1, hv, dv, dk), 7.0, device=cuda_device)
    y = torch.full((T, hv, dv), float("nan"), dtype=getattr(torch, y_dtype), device=cuda_device) if y_dtype else None
    inputs = pg.delta_inputs(q, k, v, g, beta)
    pg.precog_delta_scan(inputs, off, T, bank=bank, idx=idx, states_out=states, y_out=y)
    assert pg.precog_device_status()[0] == 0
    ref_S, ref_y = _ref(q, k, v, g, beta, off, S0)
    _check(states[:, 0], ref_S, TOL_PAIR)
    if y_dtype:
        _check(y, ref_y, TOL_PAIR)
    first = states.clone()
    bad = off.clone()
    bad[5] = T + 1                                     # sequences 4 and 5
    idx[7] = 5
    pg.precog_delta_scan(inputs, bad, T, bank=bank, idx=idx, states_out=states.fill_(7.0), y_out=y)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_OFFSETS | pg.PRECOG_DEV_BAD_INDEX)
    keep = torch.ones(n, dtype=torch.bool, device=cuda_device)
    keep[[4, 5, 7]] = False
    assert torch.equal(states[keep], first[keep]) and bool((states[4:6] == 7.0).all())


CUT = [
    # lens, hv, dk, dv, bank, want_y: few sequences whose mean is long, so that they are cut (the
    # first one's mean is just too short to be)
    ([2000, 0, 1, 1100, 3000, 64], 1, 64, 64, True, True),
    ([2500, 0, 1, 4100, 3000, 64, 2400], 1, 64, 64, True, True),
    ([1500, 4000], 2, 128, 128, True, False),
    ([2777], 1, 40, 200, False, True),
    ([1024, 2048], 1, 128, 136, True, True),
]


@pytest.mark.parametrize("lens,hv,dk,dv,bank,want_y", CUT)
def test_sequences_cut_into_segments(cuda_device, lens, hv, dk, dv, bank, want_y):
    """Long sequences of a small batch beside empty and short ones; the bank itself receives the
    states (each sequence's row is its own), and the workspace held NaN."""
    import torch
    import paper_2608_02560_gb300 as pg
    n, T = len(lens), sum(lens)
    q, k, v, g, beta, off = _tensors(lens, 1, hv, dk, dv, torch.bfloat16, cuda_device, 7 + T, rate=0.02)
    inputs = pg.delta_inputs(q, k, v, g, beta)
    need = pg.precog_delta_scan_workspace_size(inputs, n, T)
    assert (need > 0) == (T // n > 1100)
    ws = torch.full((need // 4,), float("nan"), device=cuda_device)
    states = torch.randn((n, 1, hv, dv, dk), device=cuda_device)
    S0 = to_np(states[:, 0]) if bank else None
    y = torch.full((T, hv, dv), float("nan"), device=cuda_device) if want_y else None
    pg.precog_delta_scan(inputs, off, T, bank=states if bank else None, states_out=states, y_out=y, workspace=ws)
    assert pg.precog_device_status()[0] == 0
    ref_S, ref_y = _ref(q, k, v, g, beta, off, S0)
    _check(states[:, 0], ref_S, TOL_PAIR)
    if want_y:
        _check(y, ref_y, TOL_PAIR)


def test_cut_sequences_behind_bad_offsets_are_skipped(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, _ = _tensors([6000], 1, 1, 64, 64, torch.bfloat16, cuda_device, 3)
    off = torch.tensor([0, 2500, 2400, 6000], dtype=torch.int64, device=cuda_device)
    inputs = pg.delta_inputs(q, k, v, g, beta)
    assert pg.precog_delta_scan_workspace_size(inputs, 3, 6000) > 0
    s = torch.full((3, 1, 1, 64, 64), 7.0, device=cuda_device)
    pg.precog_delta_scan(inputs, off, 6000, states_out=s)
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_OFFSETS)
    ref, _ = _ref(q[:2500], k[:2500], v[:2500], g[:2500], beta[:2500], off[:2])
    _check(s[:1, 0], ref, TOL_PAIR)
    assert bool((s[1:] == 7.0).all())


@pytest.mark.parametrize("n,hk,hv,dk,dv,dtype,y_dtype", [
    (1, 1, 1, 8, 8, "float32", "float32"), (3, 2, 4, 128, 128, "bfloat16", "bfloat16"),
    (70, 1, 2, 72, 200, "bfloat16", "float32"), (5, 3, 3, 40, 24, "float32", "bfloat16")])
def test_step_matches_the_recurrence(cuda_device, n, hk, hv, dk, dv, dtype, y_dtype):
    """Tokens one by one on a table of slots, with idle rows, against one scan of them."""
    import torch
    import paper_2608_02560_gb300 as pg
    steps, L, slots_n = 3, 2, n + 4
    table = torch.randn((slots_n, L, hv, dv, dk), device=cuda_device)
    want = to_np(table)
    slots = torch.randperm(slots_n, device=cuda_device)[:n]
    if n > 2:
        slots[1] = -1
    for step in range(steps):
        q, k, v, g, beta, _ = _tensors([n], hk, hv, dk, dv, getattr(torch, dtype), cuda_device, 60 + step, strided=n > 1)
        if step == 1:
            g[0] = float("-inf")
        y = torch.full((n, hv, dv), float("nan"), dtype=getattr(torch, y_dtype), device=cuda_device)
        pg.precog_delta_step(pg.delta_inputs(q, k, v, g, beta), table, slots=slots, y_out=y, layer=1)
        for i, slot in enumerate(slots.tolist()):
            if slot < 0:
                assert bool((y[i] == 0).all())
                continue
            S, ref_y = oracle.delta_scan(to_np(q[i:i + 1]), to_np(k[i:i + 1]), to_np(v[i:i + 1]), to_np(g[i:i + 1]),
                                         to_np(beta[i:i + 1]), [0, 1], scale=dk ** -0.5, S0=want[slot:slot + 1, 1])
            want[slot, 1] = S[0]
            _check(y[i], ref_y[0], TOL_F32)
    _check(table, want, TOL_F32)
    assert pg.precog_device_status()[0] == 0


@pytest.mark.parametrize("n,hv,dk,dv,dtype,y_dtype", [
    (120, 5, 104, 72, "bfloat16", "bfloat16"), (130, 4, 40, 72, "float32", "float32"), (160, 8, 16, 8, "bfloat16", "float32")])
def test_step_of_large_batches(cuda_device, n, hv, dk, dv, dtype, y_dtype):
    """Enough rows to fill the SMs, where a thread has two rows of a state."""
    import torch
    import paper_2608_02560_gb300 as pg
    table = torch.randn((n + 2, 1, hv, dv, dk), device=cuda_device)
    before = to_np(table)
    slots = torch.randperm(n + 2, device=cuda_device)[:n]
    slots[::17] = -1
    q, k, v, g, beta, _ = _tensors([n], 1, hv, dk, dv, getattr(torch, dtype), cuda_device, 71, strided=True)
    y = torch.full((n, hv, dv), float("nan"), dtype=getattr(torch, y_dtype), device=cuda_device)
    pg.precog_delta_step(pg.delta_inputs(q, k, v, g, beta), table, slots=slots, y_out=y)
    at = slots.cpu().numpy()
    S0 = np.where((at >= 0)[:, None, None, None], before[np.maximum(at, 0), 0], 0.0)
    S, ref_y = _ref(q, k, v, g, beta, torch.arange(n + 1), S0)
    want = before.copy()
    want[at[at >= 0], 0] = S[at >= 0]
    _check(table, want, TOL_F32)
    _check(y[slots >= 0], ref_y[at >= 0], TOL_F32)
    assert bool((y[slots < 0] == 0).all()) and pg.precog_device_status()[0] == 0


@pytest.mark.parametrize("n,hk,hv,dk,dv,dtype,y_dtype", [
    (160, 2, 4, 104, 72, "float32", "bfloat16"), (320, 1, 4, 24, 8, "float32", None), (200, 4, 4, 128, 72, "bfloat16", "bfloat16")])
def test_large_batches_token_by_token(cuda_device, n, hk, hv, dk, dv, dtype, y_dtype):
    """The same of the scan: fp32 inputs, or bf16 ones of a few tokens each."""
    import torch
    import paper_2608_02560_gb300 as pg
    lens = [int(x) for x in np.random.default_rng(n).integers(0, 9, n)]
    T = sum(lens)
    q, k, v, g, beta, off = _tensors(lens, hk, hv, dk, dv, getattr(torch, dtype), cuda_device, 81, strided=True)
    bank = torch.randn((n, 1, hv, dv, dk), device=cuda_device)
    states = torch.empty_like(bank)
    y = torch.full((T, hv, dv), float("nan"), dtype=getattr(torch, y_dtype), device=cuda_device) if y_dtype else None
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, T, bank=bank, states_out=states, y_out=y)
    ref_S, ref_y = _ref(q, k, v, g, beta, off, to_np(bank[:, 0]))
    tol = TOL_F32 if dtype == "float32" else TOL_PAIR
    _check(states[:, 0], ref_S, tol)
    if y_dtype:
        _check(y, ref_y, tol)
    assert pg.precog_device_status()[0] == 0


def test_step_with_slots_outside_the_table(cuda_device):
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, _ = _tensors([3], 1, 1, 64, 64, torch.float32, cuda_device, 71)
    table = torch.randn((2, 1, 1, 64, 64), device=cuda_device)
    before = table.clone()
    y = torch.full((3, 1, 64), 5.0, device=cuda_device)
    pg.precog_delta_step(pg.delta_inputs(q, k, v, g, beta), table, y_out=y,
                         slots=torch.tensor([2, 0, -7], device=cuda_device))
    assert pg.precog_device_status() == (5, pg.PRECOG_DEV_BAD_INDEX)
    assert torch.equal(table[1], before[1]) and not torch.equal(table[0], before[0])
    assert bool((y[0] == 0).all()) and bool((y[2] == 0).all()) and bool((y[1] != 0).any())


def test_other_streams_and_graphs(cuda_device):
    """A scan, a step and their replay on a stream that is not the tensors' own."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, off = _tensors([100, 40], 2, 2, 128, 128, torch.bfloat16, cuda_device, 81)
    inputs = pg.delta_inputs(q, k, v, g, beta)
    tok = pg.delta_inputs(q[:2], k[:2], v[:2], g[:2], beta[:2])
    s, ref = (torch.zeros((2, 1, 2, 128, 128), device=cuda_device) for _ in range(2))
    y, ref_y = (torch.zeros((2, 2, 128), device=cuda_device) for _ in range(2))
    pg.precog_delta_scan(inputs, off, 140, states_out=ref)
    pg.precog_delta_step(tok, ref, y_out=ref_y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pg.precog_delta_scan(inputs, off, 140, states_out=s)
        pg.precog_delta_step(tok, s, y_out=y)
    s.fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s, ref) and torch.equal(y, ref_y)
    with torch.cuda.stream(side):
        pg.precog_delta_scan(inputs, off, 140, states_out=s)
        pg.precog_delta_step(tok, s, y_out=y)
    side.synchronize()
    assert torch.equal(s, ref) and torch.equal(y, ref_y)


def test_offsets_beyond_32_bits(cuda_device):
    """Inputs whose last rows lie past 2^31 elements, and a table whose last slot does."""
    import torch
    import paper_2608_02560_gb300 as pg
    T, hv = 140, 2
    stride = 2 ** 24
    wide = torch.zeros((T - 1) * stride + 2 * hv * 64, dtype=torch.bfloat16, device=cuda_device)
    view = lambda at: wide[at:].as_strided((T, hv, 64), (stride, 64, 1))  # noqa: E731
    q0, k0, v0, g, beta, off = _tensors([T], hv, hv, 64, 64, torch.bfloat16, cuda_device, 91)
    k, v = view(0), view(hv * 64)
    k.copy_(k0)
    v.copy_(v0)
    s, ref = (torch.empty((1, 1, hv, 64, 64), device=cuda_device) for _ in range(2))
    pg.precog_delta_scan(pg.delta_inputs(None, k, v, g, beta), off, T, states_out=s)
    pg.precog_delta_scan(pg.delta_inputs(None, k0, v0, g, beta), off, T, states_out=ref)
    assert torch.equal(s, ref)
    del wide
    slots = 2 ** 31 // (hv * 64 * 64) + 8
    table = torch.zeros((slots, 1, hv, 64, 64), device=cuda_device)
    table[-1] = ref[0]
    y, ref_y = (torch.empty((1, hv, 64), device=cuda_device) for _ in range(2))
    tok = pg.delta_inputs(q0[:1], k0[:1], v0[:1], g[:1], beta[:1])
    pg.precog_delta_step(tok, table, slots=torch.tensor([slots - 1], device=cuda_device), y_out=y)
    pg.precog_delta_step(tok, ref, y_out=ref_y)
    assert torch.equal(table[-1], ref[0]) and torch.equal(y, ref_y)
