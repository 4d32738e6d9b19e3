"""fp32 queries over caches held in 8 bits: a product begins when they are there.  Definitions and bounds: test_gpu_quantised.py."""
import pytest
import torch

from test_gpu_decode import i32
from test_gpu_quantised import Problem, check, check_lse

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,G,new", [(64, 4, 1), (128, 7, 1), (256, 2, 4), (128, 4, 60), (256, 2, 130)])
@pytest.mark.parametrize("page", [0, 16])
def test_queries_that_arrive_after_the_first_keys(d, G, new, page):
    """Queries read from memory (their lines left L2 as 512 MB were written), over a short cache that was read just before."""
    p = Problem(2, G, d, [90, 3], [new, new], "fp32", page, seed=d + new, cap=0.0)
    q, off, L, cache = p.q.cuda(), i32(p.off), i32(p.L), p.cache()
    out, lse = torch.zeros_like(q), torch.zeros((p.T, 2 * G), device="cuda")
    wide = torch.empty(128 << 20, dtype=torch.float32, device="cuda")
    eo, el, to, tl = p.exact()
    for i in range(20):
        out.fill_(7.0)
        wide.fill_(float(i))
        for x in (*cache, off, L, *p.place.kw().values()):
            if torch.is_tensor(x):
                x.view(torch.uint8).max()
        p.dec.attend_quantised(q, off, L, *cache, out, lse=lse, **p.place.kw())
        check(out.cpu(), eo, to, "out")
        check_lse(lse.cpu(), el, tl)
