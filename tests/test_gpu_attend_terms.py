"""Attention weights over bf16 caches that multiply V as two bf16 terms: calls of few rows, and tiles whose rows may see fewer
than 512 slots.  The bound is that of two terms, and where rows see few slots it is shown to notice one: a weight is within 2^-16 of itself
(the high part within 2^-8, what is left of it rounded within 2^-8 again), the output is rounded to within 2^-8.
"""
import pytest
import torch

from test_gpu_attend_growth import Call, two_terms

pytestmark = pytest.mark.gpu

# H, G, new, ctx, window
CASES = {
    "token": (2, 7, [1], [40], 0),
    "token_long": (4, 2, [1], [3000], 0),
    "ragged_tokens": (2, 6, [1, 3, 1, 1], [10, 700, 63, 129], 0),
    "prompt_from_nothing": (2, 4, [400], [0], 0),
    "prompts_over_little": (4, 2, [200, 300], [100, 5], 0),
    "window": (2, 4, [300], [2500], 100),
    "window_odd_heads": (2, 7, [200, 70], [900, 30], 511),
}


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("name", sorted(CASES))
def test_weights_in_two_terms(name, d):
    H, G, new, ctx, window = CASES[name]
    c = Call(H, G, d, ctx, new, 0.25, seed=d + 9, window=window)
    out, lse = c.run()
    planted = c.check(out, lse, two_terms)
    # (the roundings of thousands of weights average out: only rows of few slots show them)
    if min(min(n, window or n) for n in c.L) < 512:
        assert planted > 1.5, f"weights of one term would stay within {planted:.3g} of the bound"
