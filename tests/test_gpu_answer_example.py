"""The gated delta rule, head norms, single-token step and token log probabilities together: the
example's answers from retrieved states against one scan of the whole text.

Tolerances on a token's log probability, whose logits have a standard deviation of 2 (so a relative
error e of the last row moves them by about 2 e each, and the log probability by twice that):
* fp32: each of 2 layers adds a few errors of 1e-5 at most (states, products of other orders): 1e-5 * 8
  * 4, doubled for the tails of 60 tokens: 1e-3 is beyond it.
* bf16: the two ways round the same 12 activations (2 layers of 6) at 2^-9 each; where sums differ, so
  may a rounding: sqrt(12) * 2^-8 * 4 = 0.054 as a deviation, four of them for the largest of 60 tokens.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,tol", [("float32", 1e-3), ("bfloat16", 0.22)])
def test_answers_from_states_are_those_of_the_whole_text(cuda_device, dtype, tol):
    import torch
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_from_state.py")
    spec = importlib.util.spec_from_file_location("answer_from_state", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    said = []
    r = example.main(getattr(torch, dtype), device=cuda_device, say=said.append)
    assert r["status"][0] == 0 and r["found"] == r["wanted"] and len(said) == 6
    assert bool(torch.isfinite(r["given"]).all()) and bool((r["entropy"] > 0).all())
    assert float((r["given"] - r["scored"]).abs().max()) < tol
