"""Pins of the fp64 definitions behind the gated delta rule, the head norms with rotation and the
token log probabilities: closed forms and invariants that do not use the oracle's own code."""
import numpy as np
import pytest

import oracle


def _draw(T, hk, hv, dk, dv, seed):
    r = np.random.default_rng(seed)
    k = r.standard_normal((T, hk, dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return (r.standard_normal((T, hk, dk)), k, r.standard_normal((T, hv, dv)), -r.random((T, hv)), r.random((T, hv)))


def test_orthonormal_keys_recall_their_values():
    """beta = 1, no decay, orthonormal keys: the state is sum v k^T, and reading key i gives v_i."""
    n = 8
    k = np.eye(n)[:, None, :]
    v = np.random.default_rng(0).standard_normal((n, 1, 5))
    S, y = oracle.delta_scan(np.broadcast_to(k[:1], k.shape), k, v, np.zeros((n, 1)), np.ones((n, 1)), [0, n])
    np.testing.assert_allclose(S[0, 0] @ k[:, 0].T, v[:, 0].T, atol=1e-14)
    np.testing.assert_allclose(y[:, 0], np.broadcast_to(v[0, 0], (n, 5)), atol=1e-14)


def test_a_repeated_key_holds_the_last_value():
    k = np.zeros((3, 1, 4))
    k[:, 0, 2] = 1.0
    v = np.arange(6.0).reshape(3, 1, 2)
    S, _ = oracle.delta_scan(None, k, v, np.zeros((3, 1)), np.ones((3, 1)), [0, 3])
    np.testing.assert_allclose(S[0, 0, :, 2], v[2, 0], atol=0)


def test_splitting_a_sequence_changes_nothing():
    """Theorem 1's form for this recurrence: scanning [c; q] equals scanning q from c's state."""
    q, k, v, g, b = _draw(20, 2, 4, 8, 6, 1)
    S, y = oracle.delta_scan(q, k, v, g, b, [0, 20], scale=0.5)
    S1, y1 = oracle.delta_scan(q, k, v, g, b, [0, 7], scale=0.5)
    S2, y2 = oracle.delta_scan(q[7:], k[7:], v[7:], g[7:], b[7:], [0, 13], scale=0.5, S0=S1)
    np.testing.assert_array_equal(S, S2)
    np.testing.assert_array_equal(y, np.concatenate([y1[:7], y2]))


def test_zero_beta_only_decays_and_minus_infinity_forgets():
    q, k, v, g, b = _draw(4, 1, 1, 4, 4, 2)
    S0 = np.random.default_rng(3).standard_normal((1, 1, 4, 4))
    S, _ = oracle.delta_scan(None, k, v, g, np.zeros_like(b), [0, 4], S0=S0)
    np.testing.assert_allclose(S, S0 * np.exp(g.sum()), rtol=1e-13)
    g[2] = -np.inf
    A, _ = oracle.delta_scan(None, k, v, g, b, [0, 4], S0=S0)
    B, _ = oracle.delta_scan(None, k, v, g, b, [2, 4])
    np.testing.assert_array_equal(A, B)


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_keeps_norms_and_depends_on_differences(inter):
    r = np.random.default_rng(4)
    x = np.broadcast_to(r.standard_normal((2, 1, 10)), (2, 1, 10))
    ang = np.arange(9)[:, None] * np.array([1.0, 0.3, 0.01, 0.7])
    turn = lambda v, p: oracle.qk_norm_rope(v, "none", 0.0, None, np.cos(ang), np.sin(ang), [p], inter)  # noqa: E731
    a, b = x[:1], x[1:]
    dots = [float(np.sum(turn(a, i + 3) * turn(b, i))) for i in range(5)]
    np.testing.assert_allclose(dots, dots[0], rtol=1e-12)
    np.testing.assert_allclose(np.linalg.norm(turn(a, 5)), np.linalg.norm(a), rtol=1e-13)
    np.testing.assert_array_equal(turn(a, 5)[..., 8:], a[..., 8:])


def test_norms():
    x = np.array([[[3.0, 4.0]]])
    np.testing.assert_allclose(oracle.qk_norm_rope(x, "l2", 0.0), x / 5)
    np.testing.assert_allclose(oracle.qk_norm_rope(x, "rms", 0.0, np.array([1.0, 2.0])), x / np.sqrt(12.5) * [1, 2])


def test_logprobs_by_hand():
    x = np.log(np.array([[1.0, 2.0, 5.0, 2.0]]))
    lp, H, idx, best = oracle.token_logprobs(x, [3], 1.0, 3)
    p = np.array([0.1, 0.2, 0.5, 0.2])
    np.testing.assert_allclose(lp, np.log([0.2]))
    np.testing.assert_allclose(H, [-np.sum(p * np.log(p))])
    assert idx.tolist() == [[2, 1, 3]]
    np.testing.assert_allclose(np.exp(best), [[0.5, 0.2, 0.2]])
    lp, H, idx, best = oracle.token_logprobs(np.full((1, 3), -np.inf), [0], 1.0, 2)
    assert np.isnan(lp[0]) and np.isnan(H[0]) and idx.tolist() == [[0, 1]] and np.isnan(best).all()
