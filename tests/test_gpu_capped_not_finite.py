"""Scores that are NaN, capped and not: every output of a row that sees one is NaN, on every path, and no other row's.  Definitions and
bounds: test_gpu_quantised.py, test_gpu_decode.py."""
import pytest
import torch

import test_gpu_decode as full
from test_gpu_decode import i32
from test_gpu_quantised import Problem, check, check_lse

pytestmark = pytest.mark.gpu


# the last two: kernel launches of a call in bf16 without a cap and with one (3: the slots become bf16 in the workspace first)
PATHS = [(128, 4, 1, 2, 2), (128, 8, 4, 2, 2), (256, 2, 3, 2, 2), (64, 4, 1, 2, 2), (64, 4, 90, 2, 2), (128, 4, 90, 2, 2), (128, 4, 400, 3, 2),
         (256, 2, 200, 2, 2), (64, 4, 400, 3, 3), (256, 2, 300, 3, 3)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("d,G,new,plain,capped", PATHS)
@pytest.mark.parametrize("who", ["key", "query"])
def test_nan_scores_over_8_bits(d, G, new, plain, capped, cap, dtype, who):
    """A NaN code in a key of KV head 0, which every token of the first sequence sees; a NaN in a query of every token's first head."""
    p = Problem(2, G, d, [200, 30], [new, new], dtype, 16, seed=23, cap=cap)
    eo, el, to, tl = p.exact()
    bad = torch.zeros(p.T, 2 * G, dtype=torch.bool)
    if who == "key":
        p.code[0][0, 0, 50, 3] = 0x7f
        bad[:new, :G] = True
    else:
        p.q[:, 0, 5] = float("nan")
        bad[:, 0] = True
    out, lse = p.attend()
    assert p.dec.device_status() == 0
    assert p.dec.launches() == (2 if dtype == "fp32" else capped if cap else plain)
    assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all())
    check(out[~bad], eo[~bad], to[~bad], "out")
    check_lse(lse[~bad], el[~bad], tl[~bad])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("d,G,new", [(128, 4, 1), (64, 4, 90), (128, 4, 90), (256, 2, 200), (128, 4, 300)])
def test_nan_scores_over_the_decoders_own_type(d, G, new, cap, dtype):
    """The same over a cache of the decoder's type, with weight sums: those of KV head 0 in the first sequence are NaN as far as that
    row sees, the others are right."""
    p = full.Problem(2, G, d, [100, 30], [new, new], dtype, 16, seed=24, cap=cap)
    eo, el, ew, to, tl, tw = p.exact()
    K = p.K.clone()
    K[0, 0, 50, 3] = float("nan")
    w = torch.zeros((2, 2, p.S), device="cuda")
    out, lse = p.attend(k=K, weight=w)
    bad = torch.zeros(p.T, 2 * G, dtype=torch.bool)
    bad[:new, :G] = True
    assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all())
    full.check(p, out[~bad], eo[~bad], to[~bad], "out")
    full.check(p, lse[~bad], el[~bad], tl[~bad], "lse")
    assert bool(w[0, 0, :100].isnan().all())
    for b, h in ((0, 1), (1, 0), (1, 1)):
        full.check(p, w[b, h].cpu(), ew[b, h], tw[b, h], "key_weight")
    assert p.dec.device_status() == 0
