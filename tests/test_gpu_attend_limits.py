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


@pytest.mark.parametrize("keep", [2 ** 31 - 1, 2 ** 31 - 500, 2 ** 30 + 1, 0, -1])
def test_keeps_out_of_range_are_refused(keep):
    """On the host, before anything is launched: no array of such a size is needed."""
    p = Problem(1, 1, 64, [40], [0], "bf16", 0, seed=62)
    k, v = p.cache(p.K), p.cache(p.V)
    n, w, kept = i32([40]), torch.zeros((1, 1, 1, 40), device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    new_len = i32([-7])
    plan = kvx.kvx_evict_plan(1, 1, n.data_ptr(), w.data_ptr(), 40, keep, 0, 0, kept.data_ptr(), new_len.data_ptr(), None, 0)
    ks, vs = (ctypes.c_void_p * 1)(k.data_ptr()), (ctypes.c_void_p * 1)(v.data_ptr())
    cache = kvx.kvx_dst_kv(ctypes.cast(ks, ctypes.POINTER(ctypes.c_void_p)), ctypes.cast(vs, ctypes.POINTER(ctypes.c_void_p)), 0, 40, *k.stride()[:3], None, 0, 0, 0)
    at = ctypes.byref
    assert kvx.lib().kvx_evict(p.dec.handle, at(plan), at(cache), at(cache), None) == kvx.KVX_ERR_INVALID_ARG
    assert "keep" in kvx.kvx_last_error()
    assert p.dec.device_status() == 0 and new_len.tolist() == [-7]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("stride", [2 ** 62, 2 ** 63 - 1, 2 ** 40])
def test_weight_strides_of_any_size(dtype, stride):
    """One sequence of one KV head has one row of sums, whose stride nothing is addressed by: products of it must not wrap."""
    p = Problem(1, 4, 64, [300], [1], dtype, 0, seed=63)
    q, k, v = p.q.cuda(), p.cache(p.K), p.cache(p.V)
    out, lse, w = torch.zeros_like(q), torch.zeros((1, 4), device="cuda"), torch.zeros(p.S + 64, device="cuda")
    off, n = i32(p.off), i32(p.L)
    ks, vs = (ctypes.c_void_p * 1)(k.data_ptr()), (ctypes.c_void_p * 1)(v.data_ptr())
    cache = kvx.kvx_dst_kv(ctypes.cast(ks, ctypes.POINTER(ctypes.c_void_p)), ctypes.cast(vs, ctypes.POINTER(ctypes.c_void_p)), 0, p.S,
                           *k.stride()[:3], None, 0, 0, 0)
    tok = kvx.kvx_new_tokens(1, 1, off.data_ptr(), n.data_ptr(), None)
    opts = kvx.kvx_attend_opts(0, None, lse.data_ptr(), w.data_ptr(), stride)
    rows = [kvx.kvx_rows(t.data_ptr(), *t.stride()[:2]) for t in (q, out)]
    at = ctypes.byref
    assert kvx.lib().kvx_attend(p.dec.handle, at(tok), at(rows[0]), at(cache), 0, at(opts), at(rows[1]), None) == kvx.KVX_OK
    assert p.dec.device_status() == 0
    eo, el, ew, to, tl, tw = p.exact()
    check(p, out.cpu(), eo, to, "out")
    check_lse(lse.cpu(), el, tl)
    check(p, w[:p.S].cpu(), ew[0, 0], tw[0, 0] + 1e-30, "key_weight")
    assert not w[p.S:].any()
