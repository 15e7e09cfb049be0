"""NaN and infinity within a sequence: what comes before them is the recurrence's, what follows is not
finite where the recurrence's is not -- in chunks, in segments and token by token alike.

Tolerances are those of test_gpu_delta.py: a finite row has seen nothing of the rest."""
import numpy as np
import pytest

from tests._util import TOL_F32, rel_err, rel_err_stored, to_np
from tests.test_gpu_delta import TOL_PAIR, _ref, _tensors

pytestmark = pytest.mark.gpu


def _like(got, ref, tol):
    """Finite where the reference is, and there within the tolerance."""
    import torch
    g, fine = to_np(got), np.isfinite(ref)
    assert np.array_equal(np.isfinite(g), fine), np.argwhere(np.isfinite(g) != fine)[:5]
    err = rel_err_stored if got.dtype == torch.bfloat16 else rel_err
    assert err(g[fine], ref[fine]) < tol


def _scan(q, k, v, g, beta, off, S0, y_dtype, dev):
    import torch
    import paper_2608_02560_gb300 as pg
    T, hv, dv, dk, n = q.shape[0], v.shape[1], v.shape[2], q.shape[2], off.numel() - 1
    s = torch.full((n, 1, hv, dv, dk), 7.0, device=dev)
    y = torch.full((T, hv, dv), 7.0, dtype=y_dtype, device=dev)
    pg.precog_delta_scan(pg.delta_inputs(q, k, v, g, beta), off, T, bank=S0, states_out=s, y_out=y)
    alone = torch.full_like(s, 7.0)
    pg.precog_delta_scan(pg.delta_inputs(None, k, v, g, beta), off, T, bank=S0, states_out=alone)
    assert pg.precog_device_status()[0] == 0
    return s[:, 0], y, alone[:, 0]


BROKEN = ["k nan", "k inf", "v nan", "v inf", "v -inf", "g nan", "g inf", "beta nan", "beta inf", "bank inf"]


@pytest.mark.parametrize("what", BROKEN)
@pytest.mark.parametrize("dtype,y_dtype,lens,at,hk,hv,dk,dv", [
    ("bfloat16", "float32", [200, 130], [70], 1, 2, 128, 128),          # in the middle of a chunk
    ("bfloat16", "bfloat16", [129, 64, 200], [128, 150, 202], 2, 2, 64, 200),   # first and last tokens of a chunk
    ("bfloat16", "bfloat16", [300], [45], 1, 1, 40, 24),
    ("bfloat16", "float32", [5000], [2600], 1, 1, 64, 64),               # cut into segments
    ("float32", "float32", [200, 130], [70], 1, 2, 128, 128),            # token by token
    ("bfloat16", "bfloat16", [7, 9], [3], 1, 2, 64, 64)])
def test_what_precedes_a_broken_token_is_untouched(cuda_device, what, dtype, y_dtype, lens, at, hk, hv, dk, dv):
    import torch
    dt = getattr(torch, dtype)
    q, k, v, g, beta, off = _tensors(lens, hk, hv, dk, dv, dt, cuda_device, 5 + sum(lens), rate=0.2)
    S0 = torch.randn((len(lens), 1, hv, dv, dk), device=cuda_device)
    name, value = what.split()
    value = float(value)
    for t in at:
        if name == "k":
            k[t, -1, 5] = value
        elif name == "v":
            v[t, -1, 11] = value
            v[t, 0, dv - 1] = value
        elif name == "g":
            g[t, 0] = value
        elif name == "beta":
            beta[t, -1] = value
        else:
            S0[-1, 0, 0, 3, 7] = value
    s, y, alone = _scan(q, k, v, g, beta, off, S0, getattr(torch, y_dtype), cuda_device)
    with np.errstate(invalid="ignore", over="ignore"):
        ref_S, ref_y = _ref(q, k, v, g, beta, off, to_np(S0[:, 0]))
    assert not np.isfinite(ref_S).all() and np.isfinite(ref_y).any()
    tol = TOL_F32 if dtype == "float32" else TOL_PAIR
    _like(s, ref_S, tol)
    _like(alone, ref_S, tol)
    _like(y, ref_y, tol)


@pytest.mark.parametrize("lens", [[150], [100, 64, 1, 130], [5000], [1500, 2100]])
@pytest.mark.parametrize("rate", [0.01, 0.1, 0.5, 1.5])
def test_growth_that_the_correction_holds_back(cuda_device, rate, lens):
    """Two keys by turns, beta = 1, gates that grow: each token replaces what its key holds, so the state
    stays small although the growth over a chunk or a segment is anything up to beyond fp32."""
    import torch
    q, k, v, g, beta, off = _tensors(lens, 1, 2, 64, 72, torch.bfloat16, cuda_device, 3)
    k.zero_()
    k[::2, :, 9] = 1.0
    k[1::2, :, 30] = 1.0
    g.fill_(rate)
    g[:, 1] *= torch.rand(g.shape[0], device=cuda_device).round()
    beta.fill_(1.0)
    s, y, alone = _scan(q, k, v, g, beta, off, None, torch.float32, cuda_device)
    ref_S, ref_y = _ref(q, k, v, g, beta, off)
    assert np.abs(ref_S).max() < 1e3
    for got, ref in ((s, ref_S), (alone, ref_S), (y, ref_y)):
        _like(got, ref, TOL_PAIR)


@pytest.mark.parametrize("lens,rate", [([300], 0.1), ([90, 200], 0.02), ([4000], 0.01), ([1400, 1300], 0.02)])
def test_growth_of_the_state_itself(cuda_device, lens, rate):
    """Keys that differ and betas below 1: what the keys do not touch grows with the gates."""
    import torch
    q, k, v, g, beta, off = _tensors(lens, 1, 1, 64, 136, torch.bfloat16, cuda_device, 13)
    g.fill_(rate)
    beta *= 0.2
    S0 = torch.randn((len(lens), 1, 1, 136, 64), device=cuda_device)
    s, y, alone = _scan(q, k, v, g, beta, off, S0, torch.bfloat16, cuda_device)
    ref_S, ref_y = _ref(q, k, v, g, beta, off, to_np(S0[:, 0]))
    for got, ref in ((s, ref_S), (alone, ref_S), (y, ref_y)):
        _like(got, ref, TOL_PAIR)


def test_a_bank_that_receives_the_states_of_broken_sequences(cuda_device):
    """The initial states are read again where the states go: rows that broke and rows that did not."""
    import torch
    import paper_2608_02560_gb300 as pg
    q, k, v, g, beta, off = _tensors([190, 77], 1, 2, 128, 128, torch.bfloat16, cuda_device, 15)
    v[100, 0, 17] = float("inf")
    table = torch.randn((2, 1, 2, 128, 128), device=cuda_device)
    S0 = to_np(table[:, 0])
    pg.precog_delta_scan(pg.delta_inputs(None, k, v, g, beta), off, 267, bank=table, states_out=table)
    with np.errstate(invalid="ignore", over="ignore"):
        ref_S, _ = _ref(None, k, v, g, beta, off, S0)
    _like(table[:, 0], ref_S, TOL_PAIR)
    assert pg.precog_device_status()[0] == 0


@pytest.mark.parametrize("dtype,lens,at", [("bfloat16", [200, 130], 70), ("bfloat16", [5000], 2600), ("float32", [90], 33)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_broken_query_breaks_its_own_readout_alone(cuda_device, dtype, lens, at, value):
    import torch
    q, k, v, g, beta, off = _tensors(lens, 1, 2, 64, 64, getattr(torch, dtype), cuda_device, 25, rate=0.2)
    q[at, 0, 3] = value
    s, y, alone = _scan(q, k, v, g, beta, off, None, torch.float32, cuda_device)
    with np.errstate(invalid="ignore", over="ignore"):
        ref_S, ref_y = _ref(q, k, v, g, beta, off)
    assert np.isfinite(ref_S).all() and not np.isfinite(ref_y[at]).any()
    tol = TOL_F32 if dtype == "float32" else TOL_PAIR
    for got, ref in ((s, ref_S), (alone, ref_S), (y, ref_y)):
        _like(got, ref, tol)
