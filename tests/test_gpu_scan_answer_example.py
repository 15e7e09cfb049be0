"""The causal convolution, the diagonal scan, block norms, single-token steps and adjusted logits together: the
example's answers from retrieved windows and states against one scan of the whole text.

Tolerances on a token's log probability, whose logits have a standard deviation of 2, up to 2.4 after the penalty
(so a relative error e of the last row moves them by about 2.4 e each, and the log probability by twice that):
* fp32: each of 2 layers adds some ten errors of 1e-5 at most (states, products of other orders), and a residual
  that the next layer normalises: 1e-5 * 20 * 5 = 1e-3, doubled for the tails of 60 tokens.
* bf16: the two ways round the same 17 activations (2 layers of 8, and the logits) at 2^-9 each; where sums
  differ, so may a rounding: sqrt(17) * 2^-8 * 5 = 0.08 as a deviation, four of them for the largest of 60."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,tol", [("float32", 2e-3), ("bfloat16", 0.32)])
def test_answers_from_windows_and_states_are_those_of_the_whole_text(cuda_device, dtype, tol):
    import torch
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_from_scan_state.py")
    spec = importlib.util.spec_from_file_location("answer_from_scan_state", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    said = []
    r = example.main(getattr(torch, dtype), device=cuda_device, say=said.append)
    assert r["status"][0] == 0 and r["found"] == r["wanted"] and len(said) == 6
    assert bool(torch.isfinite(r["given"]).all()) and bool(r["allowed"].all())
    assert float((r["given"] - r["scored"]).abs().max()) < tol
