"""Where prompts over an 8-bit cache change kernels: from more than 1536 rows a sequence and KV head on (heads of 256: 512) the slots become
bf16 in the workspace first, a launch more, if the cache may fit there; capped scores of heads of 128 never do."""
import math

import pytest
import torch

from test_gpu_quantised import Problem, check, check_lse, value
from test_gpu_quantised_paths import run, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("d,G,new,first", [(64, 4, 384, False), (64, 4, 385, True), (128, 4, 384, False), (128, 4, 385, True), (128, 4, 800, True),
                                           (256, 2, 256, False), (256, 2, 257, True), (256, 2, 384, True)])
def test_the_slots_that_become_bf16_first(d, G, new, first, cap):
    p = Problem(1, G, d, [333], [new], "bf16", 16, seed=new, cap=cap)
    run(p)
    assert p.dec.launches() == (3 if first and not (cap and d == 128) else 2)


@pytest.mark.parametrize("d,G,new", [(64, 4, 400), (128, 4, 400), (256, 2, 300)])
def test_a_table_one_page_too_wide(d, G, new):
    """The workspace holds 2^24 / (heads * d) slots of the call's sequences: up to there, and one page beyond."""
    slots = (16 << 20) // d
    for more, launches in ((0, 3), (16, 2)):
        p = wide(Problem(1, G, d, [100], [new], "bf16", 16, seed=d), slots + more)
        run(p)
        assert p.dec.launches() == launches


def floor(p, window, prefix):
    """What few rows' weights may be off by besides their relative bound, in the outputs' channels.  The last of a weight's three
    terms ends at 2^-23 of the largest weight times its V row's scale, c; so each slot that is seen may be off by 2^-23 c times its code.
    Codes are at most 448 and a row's largest code is above 224, so c times a code is at most twice the largest contribution (weight
    times the V row's largest): 2^-22 of that for every slot seen.  It shows in channels where the row that has nearly all the weight is nearly zero."""
    K, V = (value(c, s).double() for c, s in zip(p.code, p.byte))
    out = torch.zeros(p.T, p.H * p.G, 1, dtype=torch.float64)
    for b, n in enumerate(p.new):
        L = p.L[b]
        i, j = torch.arange(L - n, L)[:, None], torch.arange(L)
        seen = (j <= i) & ((i - j < window) if window else True)
        if prefix is not None:
            seen = seen | (j < prefix[b])
        for head in range(p.H * p.G if n else 0):
            x = p.q[p.off[b]:p.off[b + 1], head].double() @ K[b, head // p.G, :L].T * p.scale
            x = p.cap * torch.tanh(x / p.cap) if p.cap else x
            w = torch.softmax(x.masked_fill(~seen, -math.inf), -1)
            out[p.off[b]:p.off[b + 1], head, 0] = 2.0 ** -22 * seen.sum(1) * (w * V[b, head // p.G, :L].abs().amax(-1)).amax(1)
    return out


@pytest.mark.parametrize("d,G,long,singles", [(128, 4, 300, 60), (128, 2, 200, 40), (256, 4, 300, 60), (256, 2, 100, 33), (128, 7, 25, 50), (64, 4, 200, 30)])
@pytest.mark.parametrize("opt", ["plain", "window_prefix", "capped"])
def test_a_prompt_among_single_tokens(d, G, long, singles, opt):
    """The kernel goes by the mean, so the prompt's rows run in tiles of 8, 16 or 32 (heads of 64: 128): between two sequences without
    tokens, with the others' contexts from none to long."""
    ctx = [900, 5, 0] + [37 * i % 700 for i in range(singles)]
    new = [0, long, 0] + [1] * singles
    p = Problem(2, G, d, ctx, new, "bf16", 16, seed=d + long, cap=20.0 if opt == "capped" else 0.0)
    window, prefix = (90, [3 * i % 130 for i in range(len(new))]) if opt == "window_prefix" else (0, None)
    out, lse = p.attend(window, prefix)
    assert p.dec.launches() == 2 and p.dec.device_status() == 0
    eo, el, to, tl = p.exact(window, prefix)
    check(out, eo, to + (floor(p, window, prefix) if d > 64 else 0.0), "out")
    check_lse(lse, el, tl)
    assert torch.equal(p.attend(window, prefix, lse=False)[0], out), "equal calls give equal bits"
