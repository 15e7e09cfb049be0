"""Pins of the fp64 definitions behind the causal convolution, the scan's single tokens, the block norm and
the adjusted logits: closed forms and invariants that do not use the oracle's own code."""
import math

import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("K", [2, 3, 4])
def test_a_convolution_is_a_sum_of_shifted_inputs(K):
    r = np.random.default_rng(K)
    x, w = r.standard_normal((9, 3)), r.standard_normal((3, K))
    y, behind = oracle.causal_conv(x, w, [0, 9], act=False)
    for d in range(3):
        np.testing.assert_allclose(y[:, d], np.convolve(x[:, d], w[d, ::-1])[:9], atol=1e-14)
    np.testing.assert_array_equal(behind[0], x[9 - K + 1:])


def test_a_cut_sequence_continues_from_its_window():
    r = np.random.default_rng(1)
    x, w, b = r.standard_normal((7, 4)), r.standard_normal((4, 4)), r.standard_normal(4)
    whole, last = oracle.causal_conv(x, w, [0, 7], b)
    for cut in range(8):
        y0, window = oracle.causal_conv(x[:cut], w, [0, cut], b)
        y1, behind = oracle.causal_conv(x[cut:], w, [0, 7 - cut], b, windows=window)
        np.testing.assert_allclose(np.concatenate([y0, y1]), whole, atol=1e-14)
        np.testing.assert_array_equal(behind, last)


def test_silu_of_known_values():
    np.testing.assert_allclose(oracle.silu([0.0, math.log(3.0), -math.log(3.0)]),
                               [0.0, 0.75 * math.log(3.0), -0.25 * math.log(3.0)], atol=1e-15)


@pytest.mark.parametrize("cplx", [False, True])
def test_steps_are_the_scan_of_one_sequence(cplx):
    r = np.random.default_rng(2)
    T, D, N = 6, 3, 16
    x, dt, B, C = r.standard_normal((T, D)), r.random((T, D)), r.standard_normal((T, N)), r.standard_normal((T, N))
    A = -r.random((D, N)) + (1j * r.standard_normal((D, N)) if cplx else 0)
    if cplx:
        ref_h, ref_y = oracle.scan_complex(x, dt, A.real, A.imag, B, [0, T], C=C, want_y=True)
    else:
        ref_h, ref_y = oracle.scan(x, dt, A, B, [0, T], C=C, want_y=True)
    h, y = np.zeros((1, D, N), dtype=A.dtype), []
    for t in range(T):
        h, yt = oracle.scan_step(x[t:t + 1], dt[t:t + 1], A, B[t:t + 1], C[t:t + 1], h)
        y.append(yt[0])
    np.testing.assert_allclose(np.array(y), np.asarray(ref_y).reshape(T, D), atol=1e-12)
    got = np.stack([h[0].real, h[0].imag], -1) if cplx else h[0]
    np.testing.assert_allclose(got.reshape(-1), np.asarray(ref_h).view(np.float64).reshape(-1), atol=1e-12)


def test_normed_groups_have_unit_mean_squares_and_the_residual_adds():
    r = np.random.default_rng(3)
    x, g, res = (r.standard_normal((5, 24)) for _ in range(3))
    out, none = oracle.block_norm(x, groups=3, eps=0.0)
    assert none is None
    np.testing.assert_allclose((out.reshape(5, 3, 8) ** 2).mean(-1), 1.0, atol=1e-14)
    out, h = oracle.block_norm(x, gate=g, gate_first=False, norm=False, residual=res, scale=0.5, out_norm=True, eps=0.0)
    np.testing.assert_allclose(2 * (h - res) * (1 + np.exp(-g)), x * g, atol=1e-13)
    np.testing.assert_allclose((out ** 2).mean(-1), 1.0, atol=1e-14)
    np.testing.assert_allclose(out[:, :1] * h, out * h[:, :1], atol=1e-13)


def test_adjustments_of_a_row_by_hand():
    z = np.array([[2.0, -2.0, 1.0, 0.5, 3.0]])
    out = oracle.adjust_logits(z, history=[[0, 1, -1, 0, 2]], count_from=[2], repetition=[2.0], frequency=[0.25],
                               presence=[1.0], biases=[[(3, 9.0), (3, 0.5)]], allowed=[{0, 1, 2, 3}])
    np.testing.assert_allclose(out, [[2 / 2 - 0.25 - 1, -4.0, 0.5 - 0.25 - 1, 1.0, -np.inf]])
