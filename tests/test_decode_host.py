"""Refusals of the calls that go on from a cache, decided on the host before CUDA is touched."""
import ctypes

import pytest

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth


@pytest.fixture(scope="module")
def lib():
    kvx.build()
    return kvx.lib()


def _desc(geom=synth.ModelGeom(2, 2, 128, 1e6), heads=12, dtype=kvx.KVX_BF16, max_position=0, scale=0.0, cap=0.0):
    return kvx.kvx_decoder_desc(kvx.model_geom(geom), heads, dtype, max_position, scale, cap)


@pytest.mark.parametrize("desc,code", [
    (_desc(synth.ModelGeom(2, 2, 96, 1e6)), kvx.KVX_ERR_UNSUPPORTED),          # head width
    (_desc(heads=13), kvx.KVX_ERR_UNSUPPORTED),                                # 13 query heads over 2 KV heads
    (_desc(heads=130), kvx.KVX_ERR_UNSUPPORTED),                               # 65 query heads a KV head
    (_desc(heads=0), kvx.KVX_ERR_INVALID_ARG),
    (_desc(synth.ModelGeom(0, 2, 128, 1e6)), kvx.KVX_ERR_INVALID_ARG),
    (_desc(synth.ModelGeom(2, 0, 128, 1e6)), kvx.KVX_ERR_INVALID_ARG),
    (_desc(synth.ModelGeom(2, 2, 128, 1e6, rotary_dim=24)), kvx.KVX_ERR_INVALID_ARG),
    (_desc(synth.ModelGeom(2, 2, 128, 1e6, rope_type=7)), kvx.KVX_ERR_INVALID_ARG),
    (_desc(dtype=2), kvx.KVX_ERR_INVALID_ARG),
    (_desc(max_position=-1), kvx.KVX_ERR_INVALID_ARG),
    (_desc(scale=-1.0), kvx.KVX_ERR_INVALID_ARG),
    (_desc(scale=float("nan")), kvx.KVX_ERR_INVALID_ARG),
    (_desc(cap=-0.5), kvx.KVX_ERR_INVALID_ARG),
    (_desc(cap=float("inf")), kvx.KVX_ERR_INVALID_ARG),
])
def test_create_refuses(lib, desc, code):
    h = ctypes.c_void_p()
    assert lib.kvx_decoder_create(ctypes.byref(desc), ctypes.byref(h)) == code
    assert h.value is None and kvx.kvx_last_error()


def test_null_arguments(lib):
    h = ctypes.c_void_p()
    assert lib.kvx_decoder_create(None, ctypes.byref(h)) == kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_decoder_create(ctypes.byref(_desc()), None) == kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_append(None, None, None, None, None, None, None, 0, None) == kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_attend(None, None, None, None, 0, None, None, None) == kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_evict(None, None, None, None, None) == kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_decoder_status(None, None, None, 0) == kvx.KVX_ERR_INVALID_ARG
    assert lib.kvx_decoder_launches(None) == 0
    assert lib.kvx_decoder_destroy(None) == kvx.KVX_OK
