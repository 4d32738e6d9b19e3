"""kvx: GB300-native cross-model KV translation.

Thin ctypes binding of libkvx.so (C ABI in include/kvx.h).  Functions keep the
C names; they only marshal arguments (torch tensors -> device pointers,
Python values -> C structs).  Every step of the translation runs in the
library's CUDA kernels; there is no host fallback.  If the library has not
been built, loading it raises.

The translated operator is the paper's KV^_B(C) = T_theta(KV_A(C))
(Sections 4-5): layer alignment, token-span alignment, undo source RoPE,
per-KV-head projection with GQA regrouping, target RoPE, target cache write.
"""
from __future__ import annotations

import array
import ctypes
import os
import struct
import types
from typing import Optional, Sequence

from . import _build

KVX_OK, KVX_ERR_INVALID_ARG, KVX_ERR_UNSUPPORTED, KVX_ERR_CUDA, KVX_ERR_OOM, KVX_ERR_DEVICE_STATUS = range(6)
KVX_BF16, KVX_FP32 = 0, 1
KVX_PATH_AUTO, KVX_PATH_SIMT, KVX_PATH_TCGEN05 = 0, 1, 2
KVX_DEV_SPAN_CLAMPED = 0x01
KVX_DEV_POS_CLAMPED = 0x02
KVX_DEV_PAGE_INVALID = 0x04
KVX_DEV_SEQ_CLAMPED = 0x08
KVX_DEV_WAIT_TIMEOUT = 0x10
KVX_MAX_TARGET_LAYERS = 128

I32P = ctypes.POINTER(ctypes.c_int32)
VP = ctypes.c_void_p


KVX_ROPE_DEFAULT, KVX_ROPE_LINEAR, KVX_ROPE_LLAMA3 = 0, 1, 2


class kvx_model_geom(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rope_base", ctypes.c_double),
                ("rope_type", ctypes.c_int32), ("rope_factor", ctypes.c_double),
                ("rope_low_freq_factor", ctypes.c_double), ("rope_high_freq_factor", ctypes.c_double),
                ("rope_original_max_position", ctypes.c_int32), ("rotary_dim", ctypes.c_int32)]


def model_geom(g) -> kvx_model_geom:
    """kvx_model_geom from any object with the same attribute names (the RoPE schedule and
    rotary_dim attributes are optional and default to the plain schedule over the whole head)."""
    return kvx_model_geom(g.num_layers, g.num_kv_heads, g.head_dim, g.rope_base,
                          int(getattr(g, "rope_type", 0)), float(getattr(g, "rope_factor", 1.0)),
                          float(getattr(g, "rope_low_freq_factor", 1.0)),
                          float(getattr(g, "rope_high_freq_factor", 4.0)),
                          int(getattr(g, "rope_original_max_position", 8192)),
                          int(getattr(g, "rotary_dim", 0)))


KVX_FORM_GROUPED, KVX_FORM_DENSE = 0, 1


class kvx_translator_desc(ctypes.Structure):
    _fields_ = [("src", kvx_model_geom), ("dst", kvx_model_geom), ("layer_map", I32P),
                ("dtype", ctypes.c_int32), ("max_position", ctypes.c_int32), ("path", ctypes.c_int32),
                ("form", ctypes.c_int32), ("layers_per_target", ctypes.c_int32)]


class kvx_src_kv(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_seq", ctypes.c_int32),
                ("k", ctypes.POINTER(VP)), ("v", ctypes.POINTER(VP)),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_s", ctypes.c_int64),
                ("seq_len", VP), ("pos", VP)]


class kvx_tgt_tokens(ctypes.Structure):
    _fields_ = [("total_tokens", ctypes.c_int32), ("seq_off", VP), ("span_lo", VP), ("span_hi", VP),
                ("pos", VP)]


class kvx_dst_kv(ctypes.Structure):
    _fields_ = [("k", ctypes.POINTER(VP)), ("v", ctypes.POINTER(VP)), ("paged", ctypes.c_int32),
                ("max_seq", ctypes.c_int32),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_t", ctypes.c_int64),
                ("page_table", VP), ("max_pages_per_seq", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32)]


class kvx_decoder_desc(ctypes.Structure):
    _fields_ = [("model", kvx_model_geom), ("num_q_heads", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("max_position", ctypes.c_int32), ("scale", ctypes.c_double), ("score_cap", ctypes.c_double)]


class kvx_rows(ctypes.Structure):
    _fields_ = [("ptr", VP), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class kvx_new_tokens(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("total_tokens", ctypes.c_int32), ("seq_off", VP), ("kv_len", VP),
                ("pos", VP)]


class kvx_attend_opts(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("prefix_len", VP), ("lse", VP), ("key_weight", VP),
                ("weight_stride", ctypes.c_int64)]


class kvx_evict_plan(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_layers", ctypes.c_int32), ("kv_len", VP), ("key_weight", VP),
                ("weight_stride", ctypes.c_int64), ("keep", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("recent", ctypes.c_int32), ("kept", VP), ("new_len", VP), ("kept_weight", VP),
                ("kept_weight_stride", ctypes.c_int64)]


class kvx_quantised_kv(ctypes.Structure):
    _fields_ = [("codes", kvx_dst_kv), ("k_scale", VP), ("v_scale", VP), ("scale_stride_b", ctypes.c_int64),
                ("scale_stride_h", ctypes.c_int64)]


class kvx_translator_info(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int32), ("group_in", ctypes.c_int32), ("n_tile", ctypes.c_int32),
                ("smem_bytes", ctypes.c_int32), ("threads", ctypes.c_int32), ("num_sms", ctypes.c_int32),
                ("weight_bytes", ctypes.c_int64), ("table_bytes", ctypes.c_int64)]


EXPORTS = ["kvx_translator_create", "kvx_translator_create_low_rank", "kvx_translate", "kvx_fit_create",
           "kvx_fit_accumulate", "kvx_fit_solve", "kvx_fit_reset", "kvx_fit_tokens", "kvx_fit_destroy", "kvx_build_alignment", "kvx_layer_map_nearest",
           "kvx_get_device_status", "kvx_get_info", "kvx_launches_per_translate", "kvx_last_error",
           "kvx_destroy", "kvx_translate_static", "kvx_static_last_error", "kvx_span_plan_stats",
           "kvx_enable_peer", "kvx_translate_to_device", "kvx_debug_stall_next_translate", "kvx_decoder_create",
           "kvx_decoder_destroy", "kvx_append", "kvx_attend", "kvx_evict", "kvx_decoder_status", "kvx_decoder_launches",
           "kvx_append_quantised", "kvx_attend_quantised", "kvx_quantise", "kvx_dequantise"]
KVX_PEER_STORES, KVX_PEER_STAGED = 0, 1
KVX_STATIC_SCRATCH_BYTES = 8 << 20
KVX_MAX_ATTEND_BATCH = 1024   # sequences of one kvx_attend call

_lib = None


class KvxError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"kvx status {status}: {msg}")
        self.status = status


def library_path() -> str:
    return _build.LIB


def build(force: bool = False) -> str:
    return _build.build(force=force)


def lib():
    """Load libkvx.so (raises if it was not built)."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(f"libkvx.so not built ({path}); run paper_2608_30963_gb300.build()")
        L = ctypes.CDLL(path)
        L.kvx_translator_create.argtypes = [ctypes.POINTER(kvx_translator_desc), VP, VP, ctypes.c_int32,
                                            ctypes.POINTER(VP)]
        L.kvx_translator_create_low_rank.argtypes = [ctypes.POINTER(kvx_translator_desc), ctypes.c_int32, VP, VP,
                                                     VP, VP, ctypes.c_int32, ctypes.POINTER(VP)]
        L.kvx_translate.argtypes = [VP, ctypes.POINTER(kvx_src_kv), ctypes.POINTER(kvx_tgt_tokens),
                                    ctypes.POINTER(kvx_dst_kv), VP]
        L.kvx_build_alignment.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, VP, VP, VP, VP, VP, VP,
                                          VP, VP]
        L.kvx_layer_map_nearest.argtypes = [ctypes.c_int32, ctypes.c_int32, I32P]
        L.kvx_get_device_status.argtypes = [VP, VP, ctypes.POINTER(ctypes.c_uint32), ctypes.c_int32]
        L.kvx_get_info.argtypes = [VP, ctypes.POINTER(kvx_translator_info)]
        L.kvx_launches_per_translate.argtypes = [VP]
        L.kvx_launches_per_translate.restype = ctypes.c_int32
        L.kvx_last_error.restype = ctypes.c_char_p
        L.kvx_destroy.argtypes = [VP]
        L.kvx_translate_static.argtypes = [ctypes.POINTER(kvx_translator_desc), VP, VP, ctypes.POINTER(kvx_src_kv),
                                           ctypes.POINTER(kvx_tgt_tokens), ctypes.POINTER(kvx_dst_kv),
                                           ctypes.POINTER(ctypes.c_uint32), VP]
        L.kvx_static_last_error.restype = ctypes.c_char_p
        L.kvx_fit_create.argtypes = [ctypes.POINTER(kvx_translator_desc), ctypes.c_double, ctypes.c_int32,
                                     ctypes.POINTER(VP)]
        L.kvx_fit_accumulate.argtypes = [VP, ctypes.POINTER(kvx_src_kv), ctypes.POINTER(kvx_tgt_tokens),
                                         ctypes.POINTER(kvx_dst_kv), VP]
        L.kvx_fit_solve.argtypes = [VP, VP, VP, ctypes.POINTER(ctypes.c_uint32), VP]
        L.kvx_fit_reset.argtypes = [VP, VP]
        L.kvx_fit_tokens.argtypes = [VP]
        L.kvx_fit_tokens.restype = ctypes.c_int64
        L.kvx_fit_destroy.argtypes = [VP]
        L.kvx_span_plan_stats.argtypes = [VP, VP, ctypes.POINTER(ctypes.c_int64)]
        L.kvx_enable_peer.argtypes = [ctypes.c_int32]
        L.kvx_debug_stall_next_translate.argtypes = [VP, ctypes.c_int32, ctypes.c_int32]
        L.kvx_translate_to_device.argtypes = [VP, ctypes.POINTER(kvx_src_kv), ctypes.POINTER(kvx_tgt_tokens),
                                              ctypes.POINTER(kvx_dst_kv), ctypes.c_int32, ctypes.c_int32,
                                              ctypes.POINTER(kvx_dst_kv), VP]
        L.kvx_decoder_create.argtypes = [ctypes.POINTER(kvx_decoder_desc), ctypes.POINTER(VP)]
        L.kvx_decoder_destroy.argtypes = [VP]
        # struct pointers as void*: ctypes structures by reference, or their bytes
        L.kvx_append.argtypes = [VP, VP, VP, VP, VP, VP, VP, ctypes.c_int32, VP]
        L.kvx_attend.argtypes = [VP, VP, VP, VP, ctypes.c_int32, VP, VP, VP]
        L.kvx_evict.argtypes = [VP, VP, VP, VP, VP]
        L.kvx_append_quantised.argtypes = L.kvx_append.argtypes
        L.kvx_attend_quantised.argtypes = L.kvx_attend.argtypes
        L.kvx_quantise.argtypes = L.kvx_dequantise.argtypes = [VP, ctypes.c_int32, ctypes.c_int32, VP, VP, VP, VP]
        L.kvx_decoder_status.argtypes = [VP, VP, ctypes.POINTER(ctypes.c_uint32), ctypes.c_int32]
        L.kvx_decoder_launches.argtypes = [VP]
        L.kvx_decoder_launches.restype = ctypes.c_int32
        for name in EXPORTS:
            if name not in ("kvx_last_error", "kvx_launches_per_translate", "kvx_static_last_error",
                            "kvx_fit_tokens", "kvx_decoder_launches"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def kvx_last_error() -> str:
    return lib().kvx_last_error().decode()


def _check(status: int):
    if status != KVX_OK:
        raise KvxError(status, kvx_last_error())


# --------------------------------------------------------------------------- raw C calls
def kvx_layer_map_nearest(src_layers: int, dst_layers: int):
    out = (ctypes.c_int32 * dst_layers)()
    _check(lib().kvx_layer_map_nearest(src_layers, dst_layers, out))
    return list(out)


def kvx_translator_create(desc: kvx_translator_desc, w_k_ptr: int, w_v_ptr: int, weights_on_device: bool) -> int:
    h = VP()
    _check(lib().kvx_translator_create(ctypes.byref(desc), VP(w_k_ptr), VP(w_v_ptr), int(weights_on_device),
                                       ctypes.byref(h)))
    return h.value


def kvx_translator_create_low_rank(desc: kvx_translator_desc, rank: int, a_k_ptr: int, b_k_ptr: int, a_v_ptr: int,
                                   b_v_ptr: int, weights_on_device: bool) -> int:
    h = VP()
    _check(lib().kvx_translator_create_low_rank(ctypes.byref(desc), int(rank), VP(a_k_ptr), VP(b_k_ptr),
                                                VP(a_v_ptr), VP(b_v_ptr), int(weights_on_device), ctypes.byref(h)))
    return h.value


def kvx_translate(handle: int, src: kvx_src_kv, tgt: kvx_tgt_tokens, dst: kvx_dst_kv, stream: int = 0):
    _check(lib().kvx_translate(VP(handle), ctypes.byref(src), ctypes.byref(tgt), ctypes.byref(dst), VP(stream)))


def kvx_build_alignment(batch, total_src, total_tgt, src_seq_off, src_end, tgt_seq_off, tgt_end, span_lo, span_hi,
                        dev_status=0, stream: int = 0):
    _check(lib().kvx_build_alignment(batch, total_src, total_tgt, VP(src_seq_off), VP(src_end), VP(tgt_seq_off),
                                     VP(tgt_end), VP(span_lo), VP(span_hi), VP(dev_status), VP(stream)))


def kvx_translate_static(desc: kvx_translator_desc, w_k_ptr: int, w_v_ptr: int, src: kvx_src_kv,
                         tgt: kvx_tgt_tokens, dst: kvx_dst_kv, stream: int = 0, read_status: bool = False) -> int:
    """Allocation-free translation (see include/kvx.h).  Returns the device status word when
    read_status is set (the call then synchronises the stream), else 0."""
    bits = ctypes.c_uint32(0)
    st = lib().kvx_translate_static(ctypes.byref(desc), VP(w_k_ptr), VP(w_v_ptr), ctypes.byref(src),
                                    ctypes.byref(tgt), ctypes.byref(dst),
                                    ctypes.byref(bits) if read_status else None, VP(stream))
    if st not in (KVX_OK, KVX_ERR_DEVICE_STATUS):
        raise KvxError(st, lib().kvx_static_last_error().decode())
    return bits.value


def kvx_get_device_status(handle: int, stream: int = 0, clear: bool = True) -> int:
    bits = ctypes.c_uint32(0)
    st = lib().kvx_get_device_status(VP(handle), VP(stream), ctypes.byref(bits), int(clear))
    if st not in (KVX_OK, KVX_ERR_DEVICE_STATUS):
        _check(st)
    return bits.value


def kvx_get_info(handle: int) -> kvx_translator_info:
    info = kvx_translator_info()
    _check(lib().kvx_get_info(VP(handle), ctypes.byref(info)))
    return info


def kvx_launches_per_translate(handle: int) -> int:
    return lib().kvx_launches_per_translate(VP(handle))


def kvx_enable_peer(peer_device: int):
    _check(lib().kvx_enable_peer(peer_device))


def kvx_translate_to_device(handle: int, src: kvx_src_kv, tgt: kvx_tgt_tokens, dst: kvx_dst_kv, dst_device: int,
                            mode: int, staging: Optional[kvx_dst_kv] = None, stream: int = 0):
    _check(lib().kvx_translate_to_device(VP(handle), ctypes.byref(src), ctypes.byref(tgt), ctypes.byref(dst),
                                         dst_device, mode, None if staging is None else ctypes.byref(staging),
                                         VP(stream)))


def kvx_span_plan_stats(handle: int, stream: int = 0) -> dict:
    c = (ctypes.c_int64 * 4)()
    _check(lib().kvx_span_plan_stats(VP(handle), VP(stream), c))
    return {"subtiles": c[0], "staged_tokens": c[1], "global_tokens": c[2], "subtiles_with_global": c[3]}


def kvx_destroy(handle: int):
    _check(lib().kvx_destroy(VP(handle)))


# --------------------------------------------------------------------------- torch marshalling
def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _ptr_array(tensors: Sequence) -> ctypes.Array:
    # A call passes up to four of these, one entry a layer, so on short prompts this loop is most of the
    # host's work: the pointers go through an array of 64-bit words (28 layers: 5 us; 14 us as ctypes values), and
    # through the tensor type's own data_ptr where that is a method in C (a subclass may have one of its own).
    data_ptr = getattr(type(tensors[0]), "data_ptr", None) if len(tensors) else None
    try:
        words = array.array("Q", map(data_ptr if type(data_ptr) is types.MethodDescriptorType else _ptr, tensors))
    except TypeError:   # layers without a cache (None), or objects of several types
        words = array.array("Q", map(_ptr, tensors))
    return (VP * len(words)).from_buffer(words) if words else (VP * 0)()


def _stream(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return int(getattr(stream, "cuda_stream", stream))


def _call_structs(src_k, src_v, src_seq_len, tgt_seq_off, total_tokens, dst_k, dst_v, span_lo, span_hi, src_pos,
                  tgt_pos, page_table, page_size, num_pages):
    """The three call structs of kvx_translate / kvx_fit_accumulate for torch tensors."""
    s0 = src_k[0]
    src = kvx_src_kv(s0.shape[0], s0.shape[2], _ptr_array(src_k), _ptr_array(src_v),
                     s0.stride(0), s0.stride(1), s0.stride(2), _ptr(src_seq_len), _ptr(src_pos))
    tgt = kvx_tgt_tokens(int(total_tokens), _ptr(tgt_seq_off), _ptr(span_lo), _ptr(span_hi), _ptr(tgt_pos))
    d0 = dst_k[0]
    if page_table is None:
        dst = kvx_dst_kv(_ptr_array(dst_k), _ptr_array(dst_v), 0, d0.shape[2], d0.stride(0), d0.stride(1),
                         d0.stride(2), None, 0, 0, 0)
    else:
        dst = kvx_dst_kv(_ptr_array(dst_k), _ptr_array(dst_v), 1, 0, 0, 0, 0, _ptr(page_table),
                         page_table.shape[1], page_size, num_pages or d0.shape[0])
    return src, tgt, dst


def _desc(src_geom, dst_geom, layer_map, dtype, max_position, path, form, layers_per_target, keep: list):
    lm = None
    if layer_map is not None:
        flat = [int(x) for row in layer_map for x in (row if hasattr(row, "__len__") else [row])]
        arr = (ctypes.c_int32 * len(flat))(*flat)
        keep.append(arr)
        lm = ctypes.cast(arr, I32P)
    return kvx_translator_desc(model_geom(src_geom), model_geom(dst_geom), lm, dtype, max_position, path, form,
                               layers_per_target)


class Fitter:
    """Owns one kvx_fitter: closed-form ridge fit of a linear translator's W_K, W_V from
    calibration batches (source caches and the target model's own caches of the same contexts)."""

    def __init__(self, src_geom, dst_geom, lam: float, layer_map: Optional[Sequence] = None, dtype: int = KVX_BF16,
                 form: int = KVX_FORM_GROUPED, layers_per_target: int = 1, chunk_tokens: int = 0,
                 max_position: int = 0):
        self._keep = []
        self.desc = _desc(src_geom, dst_geom, layer_map, dtype, max_position, KVX_PATH_AUTO, form, layers_per_target,
                          self._keep)
        h = VP()
        _check(lib().kvx_fit_create(ctypes.byref(self.desc), float(lam), int(chunk_tokens), ctypes.byref(h)))
        self.handle = h.value

    def accumulate(self, src_k: Sequence, src_v: Sequence, src_seq_len, tgt_seq_off, total_tokens: int,
                   tgt_k: Sequence, tgt_v: Sequence, *, span_lo=None, span_hi=None, src_pos=None, tgt_pos=None,
                   page_table=None, page_size: int = 16, num_pages: int = 0, stream=None):
        """Arguments as Translator.translate; tgt_k/tgt_v are the target model's own caches (read)."""
        src, tgt, dst = _call_structs(src_k, src_v, src_seq_len, tgt_seq_off, total_tokens, tgt_k, tgt_v, span_lo,
                                      span_hi, src_pos, tgt_pos, page_table, page_size, num_pages)
        _check(lib().kvx_fit_accumulate(VP(self.handle), ctypes.byref(src), ctypes.byref(tgt), ctypes.byref(dst),
                                        VP(_stream(stream))))

    def solve(self, w_k, w_v, stream=None) -> int:
        """Writes W_K, W_V (device tensors [L_t, H_t, in, out] of the cache dtype); returns the status word."""
        bits = ctypes.c_uint32(0)
        st = lib().kvx_fit_solve(VP(self.handle), VP(_ptr(w_k)), VP(_ptr(w_v)), ctypes.byref(bits),
                                 VP(_stream(stream)))
        if st not in (KVX_OK, KVX_ERR_DEVICE_STATUS):
            _check(st)
        return bits.value

    def reset(self, stream=None):
        _check(lib().kvx_fit_reset(VP(self.handle), VP(_stream(stream))))

    def tokens(self) -> int:
        return lib().kvx_fit_tokens(VP(self.handle))

    def close(self):
        if getattr(self, "handle", None):
            _check(lib().kvx_fit_destroy(VP(self.handle)))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Translator:
    """Owns one kvx_translator.  Weights are torch tensors (host or device)
    [L_t, H_t, in, out] of the translator dtype; they are copied at creation.
    With low_rank=(A_K, B_K, A_V, B_V) ([L_t, H_t, in, rank] and [L_t, H_t, rank, out]),
    w_k and w_v are ignored and the translator is a latent adapter.  layer_map is
    [L_t] or, with layers_per_target = k > 1, [L_t, k] (nested or flat)."""

    def __init__(self, src_geom, dst_geom, w_k, w_v, layer_map: Optional[Sequence] = None,
                 dtype: int = KVX_BF16, max_position: int = 0, path: int = KVX_PATH_AUTO,
                 form: int = KVX_FORM_GROUPED, layers_per_target: int = 1, low_rank=None):
        lm = None
        if layer_map is not None:
            flat = [int(x) for row in layer_map for x in (row if hasattr(row, "__len__") else [row])]
            self._lm = (ctypes.c_int32 * len(flat))(*flat)
            lm = ctypes.cast(self._lm, I32P)
        self.desc = kvx_translator_desc(model_geom(src_geom), model_geom(dst_geom), lm, dtype, max_position, path,
                                        form, layers_per_target)
        if low_rank is not None:
            a_k, b_k, a_v, b_v = (t.contiguous() for t in low_rank)
            self.handle = kvx_translator_create_low_rank(self.desc, a_k.shape[-1], _ptr(a_k), _ptr(b_k), _ptr(a_v),
                                                         _ptr(b_v), a_k.is_cuda)
        else:
            w_k = w_k.contiguous()
            w_v = w_v.contiguous()
            self.handle = kvx_translator_create(self.desc, _ptr(w_k), _ptr(w_v), w_k.is_cuda)
        self.src_geom, self.dst_geom = src_geom, dst_geom

    def info(self) -> kvx_translator_info:
        return kvx_get_info(self.handle)

    def launches_per_translate(self) -> int:
        return kvx_launches_per_translate(self.handle)

    def translate(self, src_k: Sequence, src_v: Sequence, src_seq_len, tgt_seq_off, total_tokens: int,
                  dst_k: Sequence, dst_v: Sequence, *, span_lo=None, span_hi=None, src_pos=None, tgt_pos=None,
                  page_table=None, page_size: int = 16, num_pages: int = 0, stream=None):
        """src_k/src_v: per source layer [B, H_s, S_max, d_s] tensors (strided, d contiguous).
        dst_k/dst_v: per target layer, contiguous [B, H_t, T_max, d_t] (page_table None) or paged pools
        [num_pages, page_size, H_t, d_t]."""
        src, tgt, dst = _call_structs(src_k, src_v, src_seq_len, tgt_seq_off, total_tokens, dst_k, dst_v, span_lo,
                                      span_hi, src_pos, tgt_pos, page_table, page_size, num_pages)
        kvx_translate(self.handle, src, tgt, dst, _stream(stream))

    def translate_to_device(self, src_k: Sequence, src_v: Sequence, src_seq_len, tgt_seq_off, total_tokens: int,
                            dst_k: Sequence, dst_v: Sequence, dst_device: int, mode: int = KVX_PEER_STORES, *,
                            staging_k: Optional[Sequence] = None, staging_v: Optional[Sequence] = None,
                            span_lo=None, span_hi=None, src_pos=None, tgt_pos=None, page_table=None,
                            page_size: int = 16, num_pages: int = 0, stream=None):
        """As translate, with the target cache on device dst_device (kvx_translate_to_device):
        mode KVX_PEER_STORES writes it from the kernels, KVX_PEER_STAGED translates into
        staging_k / staging_v (current device, same layout) and copies them over."""
        src, tgt, dst = _call_structs(src_k, src_v, src_seq_len, tgt_seq_off, total_tokens, dst_k, dst_v, span_lo,
                                      span_hi, src_pos, tgt_pos, page_table, page_size, num_pages)
        stg = None
        if staging_k is not None:
            _, _, stg = _call_structs(src_k, src_v, src_seq_len, tgt_seq_off, total_tokens, staging_k, staging_v,
                                      span_lo, span_hi, src_pos, tgt_pos, page_table, page_size, num_pages)
        self._keep = (dst, stg)
        kvx_translate_to_device(self.handle, src, tgt, dst, dst_device, mode, stg, _stream(stream))

    def debug_stall_next_translate(self, unit: int, wait_us: int):
        """Diagnostics: the next translate times out its on-chip waits (kvx_debug_stall_next_translate)."""
        _check(lib().kvx_debug_stall_next_translate(VP(self.handle), unit, wait_us))

    def span_plan_stats(self, stream=None) -> dict:
        """Token-span windows of the last translate (calls with spans only): sub-tiles, tokens staged in
        their sub-tile's window, tokens gathered from global memory."""
        return kvx_span_plan_stats(self.handle, _stream(stream))

    def device_status(self, stream=None, clear: bool = True) -> int:
        return kvx_get_device_status(self.handle, _stream(stream), clear)

    def close(self):
        if getattr(self, "handle", None):
            kvx_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def build_alignment(src_seq_off, src_end, tgt_seq_off, tgt_end, span_lo, span_hi, dev_status=None, stream=None):
    """Device int32 tensors in, span_lo/span_hi (device int32[T_total]) written."""
    batch = tgt_seq_off.shape[0] - 1
    kvx_build_alignment(batch, src_end.shape[0], tgt_end.shape[0], _ptr(src_seq_off), _ptr(src_end),
                        _ptr(tgt_seq_off), _ptr(tgt_end), _ptr(span_lo), _ptr(span_hi), _ptr(dev_status),
                        _stream(stream))


# A decoding step makes a call or two a layer, so their marshalling counts: the C structs are packed as bytes (field
# by field into ctypes structures they cost 12 us a call more).
_PACK_ROWS = struct.Struct("@Pqq").pack              # kvx_rows
_PACK_TOKENS = struct.Struct("@iiPPP").pack          # kvx_new_tokens
_PACK_OPTS = struct.Struct("@iPPPq").pack            # kvx_attend_opts
_PACK_PLAN = struct.Struct("@iiPPqiiiPPPq").pack     # kvx_evict_plan
_PACK_CACHE = struct.Struct("@PPiiqqqPiii4x").pack   # kvx_dst_kv
_PACK_QUANTISED = struct.Struct("@PPiiqqqPiii4xPPqq").pack   # kvx_quantised_kv


def _rows(t) -> bytes:
    """A [tokens, heads, head_dim] tensor (strided; channels contiguous) as kvx_rows."""
    st, sh, sc = t.stride()
    if sc != 1:
        raise ValueError("rows must be [tokens, heads, head_dim] with contiguous channels")
    return _PACK_ROWS(t.data_ptr(), st, sh)


def _cache(k: Sequence, v: Sequence, page_table, page_size: int, num_pages: int):
    """Layers of a cache (contiguous [B, H, S, d], or pools [pages, page_size, H, d] with a page table) as kvx_dst_kv, and
    what has to live as long."""
    ptrs = array.array("Q", [t.data_ptr() for t in k])
    ptrs.extend([t.data_ptr() for t in v])
    at, k0 = ptrs.buffer_info()[0], k[0]
    if page_table is None:
        sb, sh, ss, _ = k0.stride()
        return _PACK_CACHE(at, at + 8 * len(k), 0, k0.shape[2], sb, sh, ss, 0, 0, 0, 0), ptrs
    return _PACK_CACHE(at, at + 8 * len(k), 1, 0, 0, 0, 0, page_table.data_ptr(), page_table.shape[1], page_size,
                       num_pages or k0.shape[0]), ptrs


def _raw_stream(stream) -> int:
    """As _stream; the current stream without a Stream object where torch offers it."""
    if stream is None and _current_raw_stream:
        return _current_raw_stream()
    return _stream(stream)


def _find_raw_stream():
    try:
        import torch
        get, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        return lambda: get(device())
    except (ImportError, AttributeError):
        return None


_current_raw_stream = None


class Decoder:
    """Owns one kvx_decoder: the steps of a target model's decoding that touch its cache.

    geom: the target model (as for Translator); num_q_heads query heads, consecutive groups of them
    reading one KV head.  scale: factor of q.k (0 = 1 / sqrt(head_dim)).  score_cap: c > 0 caps a
    scaled score s as c * tanh(s / c).  Calls are asynchronous on `stream` (None: torch's current
    stream) and allocate nothing; cache_k / cache_v are one layer's tensors, contiguous
    [B, H, S, d], or pools [num_pages, page_size, H, d] with an int32 page_table [B, max_pages]."""

    def __init__(self, geom, num_q_heads: int, dtype: int = KVX_BF16, scale: float = 0.0, score_cap: float = 0.0,
                 max_position: int = 0):
        self.desc = kvx_decoder_desc(model_geom(geom), int(num_q_heads), dtype, max_position, float(scale), float(score_cap))
        self.geom = geom
        self._heads, self._dim, self._q_heads = self.desc.model.num_kv_heads, self.desc.model.head_dim, int(num_q_heads)
        import torch
        self._type = torch.bfloat16 if dtype == KVX_BF16 else torch.float32
        self._f32, self._i32 = torch.float32, torch.int32
        self._code_types, self._scale_types = (torch.float8_e4m3fn, torch.uint8), (torch.float8_e8m0fnu, torch.uint8)
        global _current_raw_stream
        _current_raw_stream = _current_raw_stream or _find_raw_stream()
        h = VP()
        _check(lib().kvx_decoder_create(ctypes.byref(self.desc), ctypes.byref(h)))
        self.handle = h.value

    def _fits(self, t, tokens: int, heads: int):
        """Rows of one token count, of this decoder's heads, width and type."""
        if t.shape != (tokens, heads, self._dim) or t.dtype != self._type:
            raise ValueError(f"rows must be [{tokens}, {heads}, {self._dim}] of {self._type}, got {tuple(t.shape)} of {t.dtype}")

    def _index(self, t, least: int) -> bool:
        """Is t an int32 array of so many elements or more, one behind the other?"""
        return t.dtype == self._i32 and t.shape[0] >= least and t.is_contiguous()

    def _layer(self, k, v, batch: int, page_table, page_size: int, num_pages: int):
        """One layer of a cache as kvx_dst_kv (and what has to live as long), checked: this decoder's heads, width and
        type, room for `batch` sequences, K and V alike."""
        ks, st, H, d = k.shape, k.stride(), self._heads, self._dim
        ptrs = array.array("Q", (k.data_ptr(), v.data_ptr()))
        at = ptrs.buffer_info()[0]
        alike = v.shape == ks and v.stride() == st and k.dtype == v.dtype == self._type
        if page_table is None:
            if alike and len(ks) == 4 and ks[0] >= batch and ks[1] == H and ks[3] == d and st[3] == 1:
                return _PACK_CACHE(at, at + 8, 0, ks[2], st[0], st[1], st[2], 0, 0, 0, 0), ptrs
        else:
            ts = page_table.shape
            if page_size < 1 or (alike and ks[1:] == (page_size, H, d) and k.is_contiguous() and ts[0] >= batch
                                 and page_table.dtype == self._i32 and page_table.is_contiguous()):   # (the library refuses page sizes below 1)
                return _PACK_CACHE(at, at + 8, 1, 0, 0, 0, 0, page_table.data_ptr(), ts[1], page_size, num_pages or ks[0]), ptrs
        raise ValueError(f"caches must be alike, [B, {H}, S, {d}] or pools [pages, {page_size}, {H}, {d}] with an int32 page table, of "
                         f"{self._type}, got {tuple(ks)} and {tuple(v.shape)} of {k.dtype} and {v.dtype}")

    def _code_cache(self, k, s, layers: int, at: int, batch: int, page_table, page_size: int, num_pages: int):
        """An 8-bit cache whose layers are like codes k and scales s, their pointers at `at`, as kvx_quantised_kv; None if it does not fit."""
        shape, many = k.shape, s.shape
        if len(shape) != 4 or len(many) != 3 or shape[3] != self._dim:
            return None
        n = 8 * layers
        if page_table is None:
            b, h, slots, _ = shape
            (sb, sh, ss, sc), (zb, zh, zs) = k.stride(), s.stride()
            if h != self._heads or b < batch or sc != 1 or many[0] != b or many[1] != h or many[2] != slots or (zs != 1 and slots > 1):
                return None
            return _PACK_QUANTISED(at, at + n, 0, slots, sb, sh, ss, 0, 0, 0, 0, at + 2 * n, at + 3 * n, zb, zh)
        pages, size, h, _ = shape
        if page_size >= 1 and not (size == page_size and h == self._heads and many[0] == pages and many[1] == h and many[2] == size and k.is_contiguous()
                                   and s.is_contiguous() and page_table.dtype == self._i32 and page_table.shape[0] >= batch
                                   and page_table.is_contiguous()):       # (the library refuses page sizes below 1)
            return None
        return _PACK_QUANTISED(at, at + n, 1, 0, 0, 0, 0, page_table.data_ptr(), page_table.shape[1], page_size, num_pages or pages, at + 2 * n, at + 3 * n,
                               1, 1)

    def _code_layer(self, k, v, ks, vs, batch: int, page_table, page_size: int, num_pages: int):
        """One layer of an 8-bit cache as kvx_quantised_kv (and what has to live as long), checked: as _layer, codes and scales of K and V
        alike."""
        codes, scales = self._code_types, self._scale_types
        if (k.shape == v.shape and ks.shape == vs.shape and k.dtype in codes and v.dtype in codes and ks.dtype in scales and vs.dtype in scales
                and ((v.is_contiguous() and vs.is_contiguous() and k.is_contiguous() and ks.is_contiguous())
                     or (k.stride() == v.stride() and ks.stride() == vs.stride()))):
            ptrs = array.array("Q", (k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr()))
            cache = self._code_cache(k, ks, 1, ptrs.buffer_info()[0], batch, page_table, page_size, num_pages)
            if cache is not None:
                return cache, ptrs
        raise self._not_codes(k, ks, page_size)

    def _code_layers(self, k: Sequence, v: Sequence, k_scale: Sequence, v_scale: Sequence, batch: int, page_table, page_size: int,
                     num_pages: int):
        """Layers of an 8-bit cache, all alike, as _code_layer."""
        k0, s0, n = k[0], k_scale[0], len(k)
        ok = len(v) == len(k_scale) == len(v_scale) == n
        if ok and n == 1:
            return self._code_layer(k0, v[0], s0, v_scale[0], batch, page_table, page_size, num_pages)
        ptrs = array.array("Q")
        for like, types, both in ((k0, self._code_types, (k, v)), (s0, self._scale_types, (k_scale, v_scale))):
            shape, stride, plain = like.shape, like.stride(), like.is_contiguous()
            for some in both:
                for t in some:
                    if t.shape != shape or t.dtype not in types or not (t.is_contiguous() if plain else t.stride() == stride):
                        ok = False
                ptrs.extend([t.data_ptr() for t in some])
        cache = self._code_cache(k0, s0, n, ptrs.buffer_info()[0], batch, page_table, page_size, num_pages) if ok else None
        if cache is None:
            raise self._not_codes(k0, s0, page_size)
        return cache, ptrs

    def _not_codes(self, k, s, page_size: int):
        H, d = self._heads, self._dim
        return ValueError(f"8-bit caches must be alike: codes [B, {H}, S, {d}] of float8_e4m3fn or uint8 with scales [B, {H}, S] of float8_e8m0fnu or "
                          f"uint8, or pools [pages, {page_size}, {H}, {d}] with scales [pages, {H}, {page_size}] and an int32 page table, got "
                          f"{tuple(k.shape)} of {k.dtype} with {tuple(s.shape)} of {s.dtype}")

    def _full_layers(self, k: Sequence, v: Sequence, batch: int, page_table, page_size: int, num_pages: int):
        """Layers of a cache of the decoder's type as kvx_dst_kv, checked alike."""
        first, ptrs = self._layer(k[0], v[0], batch, page_table, page_size, num_pages)
        if len(k) == len(v) == 1:
            return first, ptrs
        shape, stride, plain = k[0].shape, k[0].stride(), k[0].is_contiguous()
        ok, dtype = len(v) == len(k), self._type
        for some in (k, v):
            for t in some:
                if t.shape != shape or t.dtype != dtype or not (t.is_contiguous() if plain else t.stride() == stride):
                    ok = False
        if not ok:
            raise ValueError(f"the layers of a cache must be alike, of {dtype}: {tuple(shape)} with strides {stride}")
        return _cache(k, v, page_table, page_size, num_pages)

    def append(self, q, k, v, seq_off, kv_len, cache_k, cache_v, q_out, *, pos=None, page_table=None, page_size: int = 16,
               num_pages: int = 0, stream=None):
        """Rotate the new tokens' q [T, Hq, d] into q_out (q itself: in place) and k [T, H, d] into the cache, and
        write v into the cache.  seq_off int32[B+1]: packed tokens of each sequence; kv_len int32[B]: its
        cached tokens with the new ones; pos int32[T]: RoPE positions (None: the slots)."""
        T, H, Hq = q.shape[0], self._heads, self._q_heads
        self._fits(q, T, Hq)
        self._fits(k, T, H)
        self._fits(v, T, H)
        self._fits(q_out, T, Hq)
        B = seq_off.shape[0] - 1
        if not (self._index(seq_off, 1) and self._index(kv_len, B) and (pos is None or (self._index(pos, T) and pos.shape[0] == T))):
            raise ValueError("seq_off [B + 1], kv_len [B] and pos [tokens] must be contiguous int32")
        tok = _PACK_TOKENS(B, T, seq_off.data_ptr(), kv_len.data_ptr(), 0 if pos is None else pos.data_ptr())
        cache, _keep = self._layer(cache_k, cache_v, B, page_table, page_size, num_pages)
        st = lib().kvx_append(self.handle, tok, _rows(q), _rows(k), _rows(v), _rows(q_out), cache, 0, _raw_stream(stream))
        if st:
            _check(st)

    def attend(self, q, seq_off, kv_len, cache_k, cache_v, out, *, window: int = 0, prefix_len=None, lse=None, key_weight=None,
               page_table=None, page_size: int = 16, num_pages: int = 0, stream=None):
        """Attention of the rotated queries q [T, Hq, d] over the cache (their own rows appended before), into out
        (not q itself).
        window: slots a token sees up to its own (0: all); prefix_len int32[B]: slots every token sees;
        lse float32[T, Hq]: log-sum-exp of each row; key_weight float32[B, H, S]: has the attention weights
        each slot receives added to it (needs lse)."""
        T, Hq, B = q.shape[0], self._q_heads, seq_off.shape[0] - 1
        self._fits(q, T, Hq)
        self._fits(out, T, Hq)
        if lse is not None and not (lse.shape == (T, Hq) and lse.is_contiguous() and lse.dtype == self._f32):
            raise ValueError("lse must be contiguous float32 [tokens, query heads]")
        if key_weight is not None and not (key_weight.shape[:2] == (B, self._heads) and key_weight.is_contiguous()
                                           and key_weight.dtype == self._f32):
            raise ValueError("key_weight must be contiguous float32 [sequences, KV heads, slots]")
        if not (self._index(seq_off, 1) and self._index(kv_len, B) and (prefix_len is None or self._index(prefix_len, B))):
            raise ValueError("seq_off [B + 1], kv_len [B] and prefix_len [B] must be contiguous int32")
        tok = _PACK_TOKENS(B, T, seq_off.data_ptr(), kv_len.data_ptr(), 0)
        opts = _PACK_OPTS(window, 0 if prefix_len is None else prefix_len.data_ptr(), 0 if lse is None else lse.data_ptr(),
                          0 if key_weight is None else key_weight.data_ptr(), 0 if key_weight is None else key_weight.shape[2])
        cache, _keep = self._layer(cache_k, cache_v, B if B <= KVX_MAX_ATTEND_BATCH else 0, page_table, page_size, num_pages)
        st = lib().kvx_attend(self.handle, tok, _rows(q), cache, 0, opts, _rows(out), _raw_stream(stream))
        if st:
            _check(st)

    def evict(self, kv_len, key_weight, keep: int, src_k: Sequence, src_v: Sequence, dst_k: Sequence, dst_v: Sequence, kept, new_len, *,
              sinks: int = 0, recent: int = 0, kept_weight=None, page_table=None, dst_page_table=None, page_size: int = 16,
              num_pages: int = 0, dst_num_pages: int = 0, stream=None):
        """Cut the cache (lists of layers) down to `keep` slots per sequence, KV head and layer, by key_weight float32[L, B, H, S]:
        rows into dst_k / dst_v, their slots into kept int32[L, B, H, keep] (-1 past the end), the lengths
        into new_len int32[B] (kv_len itself: in place), the weights into kept_weight float32[L, B, H, >= keep]."""
        L, B, H = len(src_k), kv_len.shape[0], self._heads
        if not (tuple(key_weight.shape[:3]) == (L, B, H) and key_weight.is_contiguous() and key_weight.dtype == self._f32):
            raise ValueError(f"key_weight must be contiguous float32 [{L}, {B}, {H}, slots]")
        if not (tuple(kept.shape) == (L, B, H, keep) and kept.is_contiguous() and kept.dtype == self._i32):
            raise ValueError(f"kept must be contiguous int32 [{L}, {B}, {H}, {keep}]")
        if kept_weight is not None and not (tuple(kept_weight.shape[:3]) == (L, B, H) and kept_weight.is_contiguous()
                                            and kept_weight.dtype == self._f32):
            raise ValueError(f"kept_weight must be contiguous float32 [{L}, {B}, {H}, slots]")
        if not len(src_v) == len(dst_k) == len(dst_v) == L:
            raise ValueError("src_k, src_v, dst_k and dst_v must have as many layers as one another")
        if not (self._index(kv_len, B) and self._index(new_len, B) and new_len.shape[0] == B):
            raise ValueError("kv_len and new_len must be contiguous int32 [B]")
        self._layer(src_k[0], src_v[0], B, page_table, page_size, num_pages)
        self._layer(dst_k[0], dst_v[0], B, dst_page_table, page_size, dst_num_pages)
        for first, rest in ((src_k[0], (src_k, src_v)), (dst_k[0], (dst_k, dst_v))):   # one shape and strides serve all layers
            shape, stride, plain = first.shape, first.stride(), first.is_contiguous()
            for tensors in rest:
                for t in tensors:
                    if t.shape != shape or t.dtype != self._type or not (t.is_contiguous() if plain else t.stride() == stride):
                        raise ValueError(f"the layers of a cache must be alike, of {self._type}: {tuple(shape)} with strides {stride}, got "
                                         f"{tuple(t.shape)} with strides {t.stride()} of {t.dtype}")
        plan = _PACK_PLAN(B, L, kv_len.data_ptr(), key_weight.data_ptr(), key_weight.shape[3], keep, sinks, recent, kept.data_ptr(),
                          new_len.data_ptr(), _ptr(kept_weight), 0 if kept_weight is None else kept_weight.shape[3])
        src, _keep_src = _cache(src_k, src_v, page_table, page_size, num_pages)
        dst, _keep_dst = _cache(dst_k, dst_v, dst_page_table, page_size, dst_num_pages)
        _check(lib().kvx_evict(self.handle, plan, src, dst, _raw_stream(stream)))

    def append_quantised(self, q, k, v, seq_off, kv_len, cache_k, cache_v, k_scale, v_scale, q_out, *, pos=None, page_table=None,
                         page_size: int = 16, num_pages: int = 0, stream=None):
        """As append, into one layer of a cache held in 8 bits: codes cache_k, cache_v (float8_e4m3fn or uint8) [B, H, S, d] with scales
        k_scale, v_scale (float8_e8m0fnu or uint8) [B, H, S], or pools [pages, page_size, H, d] with scales [pages, H, page_size].
        A value is its code times its row's scale."""
        T, H, Hq = q.shape[0], self._heads, self._q_heads
        self._fits(q, T, Hq)
        self._fits(k, T, H)
        self._fits(v, T, H)
        self._fits(q_out, T, Hq)
        B = seq_off.shape[0] - 1
        if not (self._index(seq_off, 1) and self._index(kv_len, B) and (pos is None or (self._index(pos, T) and pos.shape[0] == T))):
            raise ValueError("seq_off [B + 1], kv_len [B] and pos [tokens] must be contiguous int32")
        tok = _PACK_TOKENS(B, T, seq_off.data_ptr(), kv_len.data_ptr(), 0 if pos is None else pos.data_ptr())
        cache, _keep = self._code_layer(cache_k, cache_v, k_scale, v_scale, B, page_table, page_size, num_pages)
        st = lib().kvx_append_quantised(self.handle, tok, _rows(q), _rows(k), _rows(v), _rows(q_out), cache, 0, _raw_stream(stream))
        if st:
            _check(st)

    def attend_quantised(self, q, seq_off, kv_len, cache_k, cache_v, k_scale, v_scale, out, *, window: int = 0, prefix_len=None, lse=None,
                         page_table=None, page_size: int = 16, num_pages: int = 0, stream=None):
        """As attend (without weight sums), over one layer of a cache held in 8 bits (as for append_quantised)."""
        T, Hq, B = q.shape[0], self._q_heads, seq_off.shape[0] - 1
        self._fits(q, T, Hq)
        self._fits(out, T, Hq)
        if lse is not None and not (lse.shape == (T, Hq) and lse.is_contiguous() and lse.dtype == self._f32):
            raise ValueError("lse must be contiguous float32 [tokens, query heads]")
        if not (self._index(seq_off, 1) and self._index(kv_len, B) and (prefix_len is None or self._index(prefix_len, B))):
            raise ValueError("seq_off [B + 1], kv_len [B] and prefix_len [B] must be contiguous int32")
        tok = _PACK_TOKENS(B, T, seq_off.data_ptr(), kv_len.data_ptr(), 0)
        opts = _PACK_OPTS(window, 0 if prefix_len is None else prefix_len.data_ptr(), 0 if lse is None else lse.data_ptr(), 0, 0)
        cache, _keep = self._code_layer(cache_k, cache_v, k_scale, v_scale, B if B <= KVX_MAX_ATTEND_BATCH else 0, page_table, page_size, num_pages)
        st = lib().kvx_attend_quantised(self.handle, tok, _rows(q), cache, 0, opts, _rows(out), _raw_stream(stream))
        if st:
            _check(st)

    def quantise(self, kv_len, src_k: Sequence, src_v: Sequence, dst_k: Sequence, dst_v: Sequence, dst_k_scale: Sequence,
                 dst_v_scale: Sequence, *, page_table=None, dst_page_table=None, page_size: int = 16, num_pages: int = 0,
                 dst_num_pages: int = 0, stream=None):
        """Slots [0, kv_len[b]) of a cache (lists of layers, as a translation leaves it) into one held in 8 bits (lists of layers, as
        for append_quantised).  kv_len int32[B]."""
        self._convert("kvx_quantise", kv_len, (src_k, src_v), page_table, num_pages, (dst_k, dst_v, dst_k_scale, dst_v_scale), dst_page_table,
                      dst_num_pages, page_size, stream)

    def dequantise(self, kv_len, src_k: Sequence, src_v: Sequence, src_k_scale: Sequence, src_v_scale: Sequence, dst_k: Sequence,
                   dst_v: Sequence, *, page_table=None, dst_page_table=None, page_size: int = 16, num_pages: int = 0, dst_num_pages: int = 0,
                   stream=None):
        """The reverse of quantise: the values of a cache held in 8 bits, in the decoder's type (exact)."""
        self._convert("kvx_dequantise", kv_len, (src_k, src_v, src_k_scale, src_v_scale), page_table, num_pages, (dst_k, dst_v), dst_page_table,
                      dst_num_pages, page_size, stream)

    def _convert(self, call: str, kv_len, src, table, pages: int, dst, dst_table, dst_pages: int, page_size: int, stream):
        B, L = kv_len.shape[0], len(src[0])
        if not self._index(kv_len, B):
            raise ValueError("kv_len must be contiguous int32 [B]")
        if L < 1 or any(len(x) != L for x in (*src, *dst)):
            raise ValueError("the caches must have as many layers as one another, one or more, in every list")
        least = B if B <= KVX_MAX_ATTEND_BATCH else 0
        a, _keep_a = (self._full_layers if len(src) == 2 else self._code_layers)(*src, least, table, page_size, pages)
        b, _keep_b = (self._full_layers if len(dst) == 2 else self._code_layers)(*dst, least, dst_table, page_size, dst_pages)
        st = getattr(lib(), call)(self.handle, B, L, kv_len.data_ptr(), a, b, _raw_stream(stream))
        if st:
            _check(st)

    def device_status(self, stream=None, clear: bool = True) -> int:
        bits = ctypes.c_uint32(0)
        st = lib().kvx_decoder_status(self.handle, _stream(stream), ctypes.byref(bits), int(clear))
        if st not in (KVX_OK, KVX_ERR_DEVICE_STATUS):
            _check(st)
        return bits.value

    def launches(self) -> int:
        """Kernel launches of the most recent call."""
        return lib().kvx_decoder_launches(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            _check(lib().kvx_decoder_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
