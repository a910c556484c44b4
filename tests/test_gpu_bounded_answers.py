"""The example's whole path: norm and rotate, prune, write, answer with rotated rows straight into the cache, weigh, evict in place."""
import os
import sys

import pytest
import torch

import token_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tokens,sequences,answer,budget", [(400, 3, 40, 170), (1500, 2, 30, 610)])
def test_answers_in_a_cache_of_bounded_size(tokens, sequences, answer, budget, fp8):
    """Outputs against plain attention over the values read back (rounded to bf16 once more, 2^-9 of each, in logits of magnitude up to ten and values up to five,
    and so is the output).  Every place against the token that is said to lie there: a key is the token's own, normed and rotated, off by half a step of its code
    (int8: 1/254 of the row's largest magnitude; e4m3: 2^-4 of the value, 2^-10/448 of the largest), by the rounding to bf16 when the prompt was rotated
    (2^-8 of a value) and when it was read (2^-8), a value row likewise."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import bounded_answers
    finally:
        sys.path.pop(0)
    out, plain, s = bounded_answers.run(tokens=tokens, keep=0.4, sequences=sequences, answer=answer, budget=budget, fp8=fp8)
    assert float((out - plain).norm() / plain.norm()) < 2.0 ** -6
    n, hkv = s["lens"], s["k"].shape[2]
    assert n < tokens - int(0.6 * tokens) + answer                       # tokens were evicted
    holds = s["holds"].cpu()
    assert holds.shape == (sequences, hkv, n) and bool((holds[..., 1:] > holds[..., :-1]).all())
    assert bool((holds[..., -bounded_answers.RECENT:] == torch.arange(tokens + answer - bounded_answers.RECENT, tokens + answer)).all())
    if hkv > 1:
        assert not torch.equal(holds[:, 0], holds[:, 1])                  # each head has its own
    last = int(s["pos"][0, -1])
    pos = torch.cat([s["pos"].cpu(), (last + 1 + torch.arange(answer, dtype=torch.int32)).expand(3, -1)], 1)
    for b in range(sequences):
        keys, values = torch.cat([s["k"][b], s["new_k"][b]]).cpu(), torch.cat([s["v"][b], s["new_v"][b]]).cpu().double()
        want, _ = ref.turned(keys, pos, s["frequencies"], s["axis"], False, s["k_norm"].cpu(), 1e-6)
        for h in range(hkv):
            at = holds[b, h]
            for got, w in ((s["cache_k"][b, :, h], want[at, h]), (s["cache_v"][b, :, h], values[at, h])):
                largest = w.abs().amax(-1, keepdim=True) * (1 + 2.0 ** -7)
                half = torch.maximum(2.0 ** -4 * w.abs(), largest * 2.0 ** -10 / 448) if fp8 else largest / 254
                excess = (got.cpu().double() - w).abs() - (half + 3 * 2.0 ** -8 * w.abs() + 2.0 ** -9 * largest)
                assert float(excess.max()) <= 0
