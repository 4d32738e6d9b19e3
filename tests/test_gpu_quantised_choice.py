"""Where prompts over an 8-bit cache change kernels: from more than 1536 rows a sequence and KV head on (heads of 256: 512) the slots become
bf16 in the workspace first, a launch more, if the cache may fit there; capped scores of heads of 128 never do."""
import pytest

from test_gpu_quantised import Problem
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


@pytest.mark.parametrize("d,G,long,singles", [(128, 4, 300, 60), (128, 2, 200, 40), (256, 4, 300, 60), (256, 2, 100, 33), (128, 7, 25, 50), (64, 4, 200, 30)])
@pytest.mark.parametrize("opt", ["plain", "window_prefix", "capped"])
def test_a_prompt_among_single_tokens(d, G, long, singles, opt):
    """The kernel goes by the mean, so the prompt's rows run in tiles of 8, 16 or 32 (heads of 64: 128): between two sequences without
    tokens, with the others' contexts from none to long."""
    ctx = [900, 5, 0] + [37 * i % 700 for i in range(singles)]
    new = [0, long, 0] + [1] * singles
    p = Problem(2, G, d, ctx, new, "bf16", 16, seed=d + long, cap=20.0 if opt == "capped" else 0.0)
    run(p, *((90, [3 * i % 130 for i in range(len(new))]) if opt == "window_prefix" else (0, None)))
    assert p.dec.launches() == 2
