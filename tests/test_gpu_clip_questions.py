"""The example's whole path: prune, write the survivors into the cache, questions and answers over it, read back."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tokens,questions", [(600, 3), (2500, 12)])
def test_questions_about_a_pruned_clip(tokens, questions, fp8):
    """Against plain attention over the values read back: those are rounded to bf16 once more (2^-9 of each, in logits of magnitude up to ten and in
    values up to five), and so is the output."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import clip_questions
    finally:
        sys.path.pop(0)
    out, plain, kept = clip_questions.run(tokens=tokens, keep=0.4, questions=questions, answer=3, fp8=fp8)
    assert kept == tokens - int(0.6 * tokens)
    assert float((out - plain).norm() / plain.norm()) < 2.0 ** -6
