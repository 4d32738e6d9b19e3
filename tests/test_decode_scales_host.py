"""Scales and caps of a decoder that 32 bits do not hold are refused on the host, before CUDA is touched."""
import ctypes

import pytest

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth


def create(scale, cap):
    kvx.build()
    h = ctypes.c_void_p()
    desc = kvx.kvx_decoder_desc(kvx.model_geom(synth.ModelGeom(2, 2, 128, 1e6)), 12, kvx.KVX_BF16, 0, scale, cap)
    st = kvx.lib().kvx_decoder_create(ctypes.byref(desc), ctypes.byref(h))
    if h.value:
        kvx.lib().kvx_decoder_destroy(h)
    return st


@pytest.mark.parametrize("scale,cap", [(1e300, 0.0), (1e-300, 0.0), (5e-324, 0.0), (1e-39, 0.0), (0.0, 1e300), (0.0, 1e-300), (0.0, 1e-39), (0.0, 3.3e38),
                                       (1e30, 1e-30), (1e-30, 1e30)])
def test_numbers_that_32_bits_do_not_hold(scale, cap):
    """As floats they would be zero or infinite: no cap, no scores, or NaN in every output."""
    assert create(scale, cap) == kvx.KVX_ERR_INVALID_ARG and "32 bits" in kvx.kvx_last_error()


@pytest.mark.parametrize("scale,cap", [(0.0, 0.0), (1.0, 50.0), (0.0, 1e-3), (0.0, 30000.0), (1e-6, 1e6), (1e6, 0.0)])
def test_numbers_that_it_holds(scale, cap):
    assert create(scale, cap) in (kvx.KVX_OK, kvx.KVX_ERR_CUDA)      # (without a device: no CUDA device)
