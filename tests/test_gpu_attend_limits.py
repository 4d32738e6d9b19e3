"""kvx_attend and kvx_evict at the ends of their arguments' ranges."""
import ctypes

import pytest
import torch

import paper_2608_30963_gb300 as kvx

from test_gpu_decode import Problem, check, check_lse, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30 + 1, 2 ** 30, 2 ** 30 - 1])
@pytest.mark.parametrize("d,new,kv_len,prefix", [(128, [400, 5], [390, 3], None), (64, [40, 300], [200, 100], [3, 7]), (256, [90, 1], [60, 1], None)])
def test_windows_wider_than_any_cache(d, new, kv_len, prefix, window, dtype):
    """As no window, also where a call's first tokens have slots below zero."""
    p = Problem(2, 4, d, [0, 0], new, dtype, 16, seed=61, kv_len=kv_len)
    w = torch.zeros((2, 2, p.S), device="cuda")
    out, lse = p.attend(window, prefix, weight=w)
    eo, el, ew, to, tl, tw = p.exact(0, prefix)
    check(p, out, eo, to, "out")
    check_lse(lse, el, tl)
    check(p, w.cpu(), ew, tw + 1e-30, "key_weight")
    base, _ = p.attend(0, prefix)
    assert torch.equal(out, base)
