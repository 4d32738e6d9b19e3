"""Keys under a scale byte of 255 (infinity; never written by the library): their values are infinities of both signs, so a score
over them is NaN, on every path.  Definitions and bounds: test_gpu_quantised.py."""
import pytest
import torch

from test_gpu_quantised import Problem, check, check_lse
from test_gpu_quantised_infinite import SIZES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("d,G,ctx,new", SIZES)
def test_keys_under_an_infinite_scale(d, G, ctx, new, cap, dtype):
    """In one slot of KV head 0 in the first sequence, which all its tokens see."""
    p = Problem(2, G, d, ctx, new, dtype, 16, seed=d + G, cap=cap)
    eo, el, to, tl = p.exact()
    p.byte[0][0, 0, ctx[0] // 2] = 255
    signs = torch.sign(p.q[:new[0], :G].double()) * torch.sign((p.code[0][0, 0, ctx[0] // 2].int() < 128).double() - 0.5)
    assert bool((signs.amax(-1) == 1).all() and (signs.amin(-1) == -1).all())
    out, lse = p.attend()
    bad = torch.zeros(p.T, 2 * G, dtype=torch.bool)
    bad[:new[0], :G] = True
    assert p.dec.device_status() == 0
    assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all())
    check(out[~bad], eo[~bad], to[~bad], "out")
    check_lse(lse[~bad], el[~bad], tl[~bad])
