"""Refusals of the calls on caches held in 8 bits that are decided on the host before CUDA is touched, and their structs."""
import ctypes

import pytest

import paper_2608_30963_gb300 as kvx


@pytest.fixture(scope="module")
def lib():
    kvx.build()
    return kvx.lib()


def test_null_arguments(lib):
    bad = kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_append_quantised(None, None, None, None, None, None, None, 0, None) == bad and "append_quantised" in kvx.kvx_last_error()
    assert lib.kvx_attend_quantised(None, None, None, None, 0, None, None, None) == bad and "attend_quantised" in kvx.kvx_last_error()
    assert lib.kvx_quantise(None, 1, 1, None, None, None, None) == bad and "quantise" in kvx.kvx_last_error()
    assert lib.kvx_dequantise(None, 1, 1, None, None, None, None) == bad and "dequantise" in kvx.kvx_last_error()


def test_the_bytes_that_the_binding_packs_are_the_structs():
    cache = kvx._PACK_QUANTISED(1, 2, 1, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14)
    assert len(cache) == ctypes.sizeof(kvx.kvx_quantised_kv)
    s = kvx.kvx_quantised_kv.from_buffer_copy(cache)
    assert (s.codes.paged, s.codes.stride_t, s.codes.num_pages, s.k_scale, s.v_scale, s.scale_stride_b, s.scale_stride_h) == (1, 6, 10, 11, 12, 13, 14)
