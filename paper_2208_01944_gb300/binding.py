"""Thin ctypes binding of libpalquant.so (include/palquant.h).

Functions keep the C names and argument order.  They only marshal arguments:
device buffers are passed as ``torch.Tensor`` (their ``data_ptr()``) or raw integer
addresses, host arrays as numpy arrays or sequences, streams as ``torch.cuda.Stream``
or raw handles (default: torch's current stream).  A non-OK status raises
:class:`PalquantError`.  The calls of the 8-bit transformer layers hold tensors against
their descriptors first and raise :class:`ArgumentError`; addresses are the caller's word.  Every computation happens in the CUDA library; if it has
not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpalquant.so")

PQ_OK, PQ_EINVAL, PQ_EUNSUPPORTED, PQ_ECUDA, PQ_ETIMEOUT = 0, -1, -2, -3, -4
PQ_CODES_INT8, PQ_CODES_E4M3, PQ_CODES_C16, PQ_CODES_C16P2, PQ_CODES_C32F4, PQ_CODES_F16 = 0, 1, 2, 3, 4, 5
PQ_F32, PQ_F16, PQ_BF16 = 0, 1, 2
PQ_LAYER_INPUTS_READY = 1  # pq_layer_desc.flags: the previous kernel on the stream writes neither input nor weights

# Every symbol include/palquant.h declares.
EXPORTS = [
    "palquant_strerror", "palquant_version", "palquant_act_steps_scratch_bytes", "palquant_act_steps",
    "palquant_act_steps_noalloc",
    "palquant_weight_steps", "palquant_epilogue_scales", "palquant_packed_weight_bytes",
    "palquant_pack_weights_host", "palquant_pack_weights", "palquant_pack_weight_codes_host",
    "palquant_unpack_weight_codes_host", "palquant_quantize_act", "palquant_group_conv", "palquant_layer_fused",
    "palquant_quantize_layer_fused",
    "palquant_sync_check", "palquant_set_wait_limit_ns", "palquant_watchdog_selftest", "palquant_conv_plan",
    "palquant_conv2d_f32", "palquant_stem_pool_f32", "palquant_maxpool2d_f32", "palquant_avgpool_f32",
    "palquant_linear_f32",
    "palquant_cyclic_shuffle_module", "palquant_bitsplit_desc", "palquant_bitsplit_scratch_bytes",
    "palquant_bitsplit_pack_weight_codes_host", "palquant_bitsplit_act", "palquant_bitsplit_conv",
    "palquant_pack_weights_odd_host", "palquant_fake_quant_forward", "palquant_fake_quant_scratch_bytes",
    "palquant_fake_quant_backward", "palquant_quantize_act_lu", "palquant_quantize_layer_fused_lu",
    "palquant_quantize_tokens", "palquant_linear_code_format", "palquant_linear_i8",
    "palquant_linear_q8_scratch_bytes", "palquant_linear_q8", "palquant_kv8_append", "palquant_kv8_read",
    "palquant_kv8_attention_scratch_bytes", "palquant_kv8_attention",
    "palquant_kv8_attention_sinks_scratch_bytes", "palquant_kv8_attention_sinks",
    "palquant_kv8_attention_tree_scratch_bytes", "palquant_kv8_attention_tree",
    "palquant_rope_turns_host", "palquant_qk_norm_rope", "palquant_w4_packed_bytes", "palquant_w4_pack",
    "palquant_w4_quantize", "palquant_w4_unpack", "palquant_linear_w4_scratch_bytes", "palquant_linear_w4",
]


class PalquantError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


class LayerDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "N", "H", "W", "G", "Cin_g", "Cout_g", "kh", "kw", "stride", "pad", "bits_a", "bits_w", "bits_out", "relu",
        "code_format", "flags", "wslices")]


class Shuffle(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("shift", ctypes.c_int32), ("perm", ctypes.POINTER(ctypes.c_int32))]


class ConvPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "supported", "mode", "rows_per_tile", "m_tiles", "tile_pitch", "n_block", "n_blocks", "k_chunk", "k_blocks",
        "taps", "weights_resident", "acc_stages", "smem_bytes")] + [("tiles", ctypes.c_int64), ("work_items", ctypes.c_int64),
                                                                     ("pointwise", ctypes.c_int32)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class LinearDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("N", "K", "x_type", "y_type")] + \
        [(n, ctypes.c_int64) for n in ("ldx", "ldw", "ldy")]


class KV8Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_pages", "page_tokens", "Hkv", "D")] + \
        [(n, ctypes.c_void_p) for n in ("k_dev", "v_dev", "k_scale_dev", "v_scale_dev")]


class KV8Tokens(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "B", "max_n", "table_pitch")] + \
        [(n, ctypes.c_int64) for n in ("k_token_stride", "k_head_stride", "v_token_stride", "v_head_stride")] + \
        [(n, ctypes.c_void_p) for n in ("cu_dev", "start_dev", "page_table_dev")]


class KV8Attn(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "B", "Hq", "max_q", "max_len", "causal", "window", "table_pitch")] + \
        [("scale", ctypes.c_float)] + \
        [(n, ctypes.c_int64) for n in ("q_token_stride", "q_head_stride", "o_token_stride", "o_head_stride")] + \
        [(n, ctypes.c_void_p) for n in ("cu_q_dev", "len_dev", "page_table_dev")]


class KV8Tree(ctypes.Structure):
    _fields_ = [("bits_dev", ctypes.c_void_p), ("pitch", ctypes.c_int64), ("words", ctypes.c_int32)]


class QKRope(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "w_type")] + [("tokens", ctypes.c_int64)] + \
        [(n, ctypes.c_int32) for n in ("Hq", "Hkv", "D", "R", "interleaved", "norm")] + [("eps", ctypes.c_float)] + \
        [(n, ctypes.c_int64) for n in ("q_token_stride", "q_head_stride", "k_token_stride", "k_head_stride",
                                       "q_out_token_stride", "q_out_head_stride", "k_out_token_stride", "k_out_head_stride")] + \
        [(n, ctypes.c_void_p) for n in ("pos_dev", "turns_dev", "q_weight_dev", "k_weight_dev")]


class W4Weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "K", "group", "s_type")]


_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_F32P = ctypes.POINTER(ctypes.c_float)


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run paper_2208_01944_gb300.build.build() (or __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    L.palquant_strerror.restype = ctypes.c_char_p
    L.palquant_strerror.argtypes = [_I32]
    L.palquant_version.restype = _I32
    L.palquant_act_steps_scratch_bytes.restype = ctypes.c_size_t
    L.palquant_act_steps_scratch_bytes.argtypes = [_I64, _I32]
    L.palquant_act_steps.restype = _I32
    L.palquant_act_steps.argtypes = [_P, _I64, _I32, _I32, _I32, _I32, _I32, _P, ctypes.c_size_t, _P, _P]
    L.palquant_act_steps_noalloc.restype = _I32
    L.palquant_act_steps_noalloc.argtypes = [_P, _I64, _I32, _I32, _I32, _I32, _I32, _P, _P]
    L.palquant_weight_steps.restype = _I32
    L.palquant_weight_steps.argtypes = [_P, ctypes.POINTER(LayerDesc), _P]
    L.palquant_epilogue_scales.restype = _I32
    L.palquant_epilogue_scales.argtypes = [_I32, _P, _P, ctypes.c_double, _P, Shuffle, _P, _P]
    L.palquant_packed_weight_bytes.restype = ctypes.c_size_t
    L.palquant_packed_weight_bytes.argtypes = [ctypes.POINTER(LayerDesc)]
    L.palquant_pack_weights_host.restype = _I32
    L.palquant_pack_weights_host.argtypes = [_P, ctypes.POINTER(LayerDesc), _P, _P, ctypes.c_size_t]
    L.palquant_pack_weights.restype = _I32
    L.palquant_pack_weights.argtypes = [_P, ctypes.POINTER(LayerDesc), _P, _P, ctypes.c_size_t, _P]
    L.palquant_pack_weight_codes_host.restype = _I32
    L.palquant_pack_weight_codes_host.argtypes = [_P, ctypes.POINTER(LayerDesc), _P, ctypes.c_size_t]
    L.palquant_unpack_weight_codes_host.restype = _I32
    L.palquant_unpack_weight_codes_host.argtypes = [_P, ctypes.POINTER(LayerDesc), _P]
    L.palquant_quantize_act.restype = _I32
    L.palquant_quantize_act.argtypes = [_P, _P, _I64, _I32, _I32, _I32, _I32, _I32, _I32, _P, _P]
    L.palquant_group_conv.restype = _I32
    L.palquant_group_conv.argtypes = [_P, _P, _P, ctypes.POINTER(LayerDesc), _P]
    L.palquant_layer_fused.restype = _I32
    L.palquant_layer_fused.argtypes = [_P, _P, ctypes.POINTER(LayerDesc), _P, _P, Shuffle, _P, _P, _P, _P, _P]
    L.palquant_quantize_layer_fused.restype = _I32
    L.palquant_quantize_layer_fused.argtypes = [_P, _P, _P, ctypes.POINTER(LayerDesc), _P, _P, Shuffle, _P, _P, _P, _P,
                                                _P]
    L.palquant_sync_check.restype = _I32
    L.palquant_sync_check.argtypes = [_P]
    L.palquant_set_wait_limit_ns.restype = _I32
    L.palquant_set_wait_limit_ns.argtypes = [ctypes.c_uint64]
    L.palquant_watchdog_selftest.restype = _I32
    L.palquant_watchdog_selftest.argtypes = [ctypes.c_uint64, _P]
    L.palquant_conv_plan.restype = _I32
    L.palquant_conv_plan.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(ConvPlan)]
    L.palquant_pack_weights_odd_host.restype = _I32
    L.palquant_pack_weights_odd_host.argtypes = [_P, ctypes.POINTER(LayerDesc), _P, _P, ctypes.c_size_t]
    L.palquant_bitsplit_desc.restype = _I32
    L.palquant_bitsplit_desc.argtypes = [ctypes.POINTER(LayerDesc), _I32, ctypes.POINTER(LayerDesc)]
    L.palquant_bitsplit_scratch_bytes.restype = ctypes.c_size_t
    L.palquant_bitsplit_scratch_bytes.argtypes = [ctypes.POINTER(LayerDesc), _I32]
    L.palquant_bitsplit_pack_weight_codes_host.restype = _I32
    L.palquant_bitsplit_pack_weight_codes_host.argtypes = [_P, ctypes.POINTER(LayerDesc), _I32, _P, ctypes.c_size_t]
    L.palquant_bitsplit_act.restype = _I32
    L.palquant_bitsplit_act.argtypes = [_P, _P, ctypes.c_size_t, ctypes.POINTER(LayerDesc), _I32, _P]
    L.palquant_bitsplit_conv.restype = _I32
    L.palquant_bitsplit_conv.argtypes = [_P, _P, ctypes.c_size_t, _P, _P, ctypes.POINTER(LayerDesc), _I32, _P]
    L.palquant_cyclic_shuffle_module.restype = _I32
    L.palquant_cyclic_shuffle_module.argtypes = [_P, _P, ctypes.POINTER(LayerDesc), _P, _P, _I32, _P, _P, _P, _P]
    for name, args in (("palquant_conv2d_f32", [_P, _P, _P, _I64] + [_I32] * 8 + [_P]),
                       ("palquant_stem_pool_f32", [_P, _P, _P, _P, _I64, _I32, _I32, _I32, _P]),
                       ("palquant_maxpool2d_f32", [_P, _P, _I64] + [_I32] * 6 + [_P]),
                       ("palquant_avgpool_f32", [_P, _P, _I64, _I32, _I32, _I32, _P]),
                       ("palquant_linear_f32", [_P, _P, _P, _I64, _I32, _I32, _P])):
        getattr(L, name).restype = _I32
        getattr(L, name).argtypes = args
    L.palquant_quantize_act_lu.restype = _I32
    L.palquant_quantize_act_lu.argtypes = [_P, _P, _I64, _I32, _I32, _I32, _I32, _I32, _I32, _P, _P, _P]
    L.palquant_quantize_layer_fused_lu.restype = _I32
    L.palquant_quantize_layer_fused_lu.argtypes = list(L.palquant_quantize_layer_fused.argtypes[:1]) + [_P, _P] + \
        list(L.palquant_quantize_layer_fused.argtypes[2:])
    L.palquant_fake_quant_forward.restype = _I32
    L.palquant_fake_quant_forward.argtypes = [_P, _P, _I64, _I32, _I32, _I32, _I32, _P, _P, _P]
    L.palquant_fake_quant_scratch_bytes.restype = ctypes.c_size_t
    L.palquant_fake_quant_scratch_bytes.argtypes = [_I64, _I32, _I32]
    L.palquant_fake_quant_backward.restype = _I32
    L.palquant_fake_quant_backward.argtypes = [_P, _P, _P, _P, _P, _I64, _I32, _I32, _I32, _I32, _P, _P, _P,
                                               ctypes.c_size_t, _P]
    L.palquant_quantize_tokens.restype = _I32
    L.palquant_quantize_tokens.argtypes = [_P, _I32, _I64, _I64, _I32, _I32, _P, _I64, _P, _P]
    L.palquant_linear_code_format.restype = _I32
    L.palquant_linear_code_format.argtypes = [ctypes.POINTER(LinearDesc)]
    L.palquant_linear_i8.restype = _I32
    L.palquant_linear_i8.argtypes = [_P, _I32, _I64, _P, _P, _P, _P, _P, _P, ctypes.POINTER(LinearDesc), _P]
    L.palquant_linear_q8_scratch_bytes.restype = ctypes.c_size_t
    L.palquant_linear_q8_scratch_bytes.argtypes = [ctypes.POINTER(LinearDesc)]
    L.palquant_linear_q8.restype = _I32
    L.palquant_linear_q8.argtypes = [_P, _P, _P, _P, _P, ctypes.POINTER(LinearDesc), _P, ctypes.c_size_t, _P]
    for name in ("palquant_kv8_append", "palquant_kv8_read"):
        getattr(L, name).restype = _I32
        getattr(L, name).argtypes = [ctypes.POINTER(KV8Cache), _P, _P, ctypes.POINTER(KV8Tokens), _P]
    L.palquant_kv8_attention_scratch_bytes.restype = ctypes.c_size_t
    L.palquant_kv8_attention_scratch_bytes.argtypes = [ctypes.POINTER(KV8Cache), ctypes.POINTER(KV8Attn)]
    L.palquant_kv8_attention.restype = _I32
    L.palquant_kv8_attention.argtypes = [ctypes.POINTER(KV8Cache), _P, _P, ctypes.POINTER(KV8Attn), _P, ctypes.c_size_t,
                                         _P]
    cache_p, attn_p, tree_p = (ctypes.POINTER(s) for s in (KV8Cache, KV8Attn, KV8Tree))
    w4_p, linear_p = ctypes.POINTER(W4Weights), ctypes.POINTER(LinearDesc)
    for name, result, args in (
            ("palquant_kv8_attention_sinks_scratch_bytes", ctypes.c_size_t, [cache_p, attn_p, _I32]),
            ("palquant_kv8_attention_sinks", _I32, [cache_p, _P, _P, attn_p, _I32, _P, ctypes.c_size_t, _P]),
            ("palquant_kv8_attention_tree_scratch_bytes", ctypes.c_size_t, [cache_p, attn_p, tree_p]),
            ("palquant_kv8_attention_tree", _I32, [cache_p, _P, _P, attn_p, tree_p, _P, ctypes.c_size_t, _P]),
            ("palquant_rope_turns_host", _I32, [_P, _I32, _P]),
            ("palquant_qk_norm_rope", _I32, [_P, _P, _P, _P, ctypes.POINTER(QKRope), _P]),
            ("palquant_w4_packed_bytes", ctypes.c_size_t, [w4_p]),
            ("palquant_w4_pack", _I32, [_P, _I64, _P, w4_p, _P, ctypes.c_size_t, _P]),
            ("palquant_w4_quantize", _I32, [_P, _I32, _I64, w4_p, _P, ctypes.c_size_t, _P]),
            ("palquant_w4_unpack", _I32, [_P, w4_p, _P, _I64, _P, _P]),
            ("palquant_linear_w4_scratch_bytes", ctypes.c_size_t, [w4_p, linear_p]),
            ("palquant_linear_w4", _I32, [_P, _P, _P, _P, w4_p, linear_p, _P, ctypes.c_size_t, _P])):
        getattr(L, name).restype = result
        getattr(L, name).argtypes = args
    return L


lib = _load()


# ----------------------------------------------------------------- marshalling
def _ptr(obj):
    """Device or host address of a tensor / array / int (None -> NULL)."""
    if obj is None or type(obj) is int:
        return obj
    address = getattr(obj, "data_ptr", None)
    if address is not None:
        assert obj.is_contiguous(), "tensors passed to libpalquant must be contiguous"
        return address()
    if isinstance(obj, np.ndarray):
        assert obj.flags["C_CONTIGUOUS"]
        return obj.ctypes.data
    if isinstance(obj, int):
        return obj
    raise TypeError(f"cannot pass {type(obj)} as a pointer")


def _strided(obj):
    """As _ptr, for a tensor whose strides are in its descriptor."""
    address = getattr(obj, "data_ptr", None)
    return address() if address is not None else _ptr(obj)


_current = None  # torch's functions for the current stream's handle and the current device, once CUDA is up


def _stream(stream):
    global _current
    if stream is None:
        if _current is None:
            import torch

            if not torch.cuda.is_initialized():
                return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
            # the handle alone: a Stream object costs 3 us a call
            _current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        return _current[0](_current[1]())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _f32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.float32))


def _check(status: int, where: str):
    if status != PQ_OK:
        raise PalquantError(status, where)


def strerror(status: int) -> str:
    return lib.palquant_strerror(status).decode()


def layer_desc(N, H, W, G, Cin_g, Cout_g, k, stride=1, pad=0, bits_a=2, bits_w=2, bits_out=2, relu=1,
               code_format=PQ_CODES_INT8, kw=None, flags=0) -> LayerDesc:
    return LayerDesc(N, H, W, G, Cin_g, Cout_g, k, k if kw is None else kw, stride, pad, bits_a, bits_w, bits_out,
                     int(relu), code_format, int(flags), 0)


def shuffle(kind=1, shift=1, perm=None):
    """pq_shuffle; the returned pair keeps the permutation array alive."""
    arr = None if perm is None else (ctypes.c_int32 * len(perm))(*[int(v) for v in perm])
    s = Shuffle(kind, shift, ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32)) if arr is not None else None)
    s._keep = arr
    return s


# ------------------------------------------------------------------ the ABI
def palquant_version() -> int:
    return lib.palquant_version()


def palquant_act_steps_scratch_bytes(P: int, G: int) -> int:
    return lib.palquant_act_steps_scratch_bytes(P, G)


def palquant_act_steps(x_dev, N, H, W, G, Cg, bits, scratch_dev, scratch_bytes, stream=None) -> np.ndarray:
    out = np.empty(G, dtype=np.float32)
    _check(lib.palquant_act_steps(_ptr(x_dev), N, H, W, G, Cg, bits, _ptr(scratch_dev), scratch_bytes, _ptr(out),
                                  _stream(stream)), "palquant_act_steps")
    return out


def palquant_act_steps_noalloc(x_dev, N, H, W, G, Cg, bits, stream=None) -> np.ndarray:
    """Per-group activation steps without any device allocation (fixed library scratch)."""
    out = np.empty(G, dtype=np.float32)
    _check(lib.palquant_act_steps_noalloc(_ptr(x_dev), N, H, W, G, Cg, bits, _ptr(out), _stream(stream)),
           "palquant_act_steps_noalloc")
    return out


def palquant_weight_steps(w_host: np.ndarray, d: LayerDesc) -> np.ndarray:
    w = _f32(w_host)
    out = np.empty(d.G, dtype=np.float32)
    _check(lib.palquant_weight_steps(_ptr(w), ctypes.byref(d), _ptr(out)), "palquant_weight_steps")
    return out


def palquant_epilogue_scales(G, s_w, s_a, alpha=1.0, s_next=None, shuf=None):
    s_w, s_a = _f32(s_w), _f32(s_a)
    sn = None if s_next is None else _f32(s_next)
    m_out = np.empty(G, dtype=np.float32)
    m_req = np.empty(G, dtype=np.float32)
    _check(lib.palquant_epilogue_scales(G, _ptr(s_w), _ptr(s_a), float(alpha), _ptr(sn), shuf or shuffle(0, 0),
                                        _ptr(m_out), _ptr(m_req)), "palquant_epilogue_scales")
    return m_out, (m_req if sn is not None else None)


def palquant_packed_weight_bytes(d: LayerDesc) -> int:
    return lib.palquant_packed_weight_bytes(ctypes.byref(d))


def palquant_pack_weights_host(w_host, d: LayerDesc, inv_sw) -> np.ndarray:
    n = palquant_packed_weight_bytes(d)
    if n == 0:
        raise PalquantError(PQ_EUNSUPPORTED, "palquant_packed_weight_bytes")
    out = np.empty(n, dtype=np.uint8)
    w, inv = _f32(w_host), _f32(inv_sw)
    _check(lib.palquant_pack_weights_host(_ptr(w), ctypes.byref(d), _ptr(inv), _ptr(out), n), "palquant_pack_weights_host")
    return out


def palquant_pack_weights(w_host, d: LayerDesc, inv_sw, packed_dev, packed_bytes, stream=None):
    w, inv = _f32(w_host), _f32(inv_sw)
    _check(lib.palquant_pack_weights(_ptr(w), ctypes.byref(d), _ptr(inv), _ptr(packed_dev), packed_bytes,
                                     _stream(stream)), "palquant_pack_weights")


def palquant_pack_weight_codes_host(wq_host, d: LayerDesc) -> np.ndarray:
    n = palquant_packed_weight_bytes(d)
    if n == 0:
        raise PalquantError(PQ_EUNSUPPORTED, "palquant_packed_weight_bytes")
    out = np.empty(n, dtype=np.uint8)
    wq = np.ascontiguousarray(wq_host, dtype=np.int8)
    _check(lib.palquant_pack_weight_codes_host(_ptr(wq), ctypes.byref(d), _ptr(out), n), "palquant_pack_weight_codes_host")
    return out


def palquant_unpack_weight_codes_host(packed_host, d: LayerDesc) -> np.ndarray:
    """[G][Cout_g][kh][kw][Cin_g], or [G][Cout_g][kh][kw][R][Cin_g] with R = d.wslices > 1 weight slices."""
    R = d.wslices if d.wslices > 1 else 1
    shape = (d.G, d.Cout_g, d.kh, d.kw, d.Cin_g) if R == 1 else (d.G, d.Cout_g, d.kh, d.kw, R, d.Cin_g)
    out = np.empty(shape, dtype=np.int8)
    pk = np.ascontiguousarray(packed_host, dtype=np.uint8)
    _check(lib.palquant_unpack_weight_codes_host(_ptr(pk), ctypes.byref(d), _ptr(out)), "palquant_unpack_weight_codes_host")
    return out


def palquant_quantize_act(x_dev, q_dev, N, H, W, G, Cg, bits, inv_s, code_format=PQ_CODES_INT8, stream=None):
    inv = _f32(inv_s)
    _check(lib.palquant_quantize_act(_ptr(x_dev), _ptr(q_dev), N, H, W, G, Cg, bits, code_format, _ptr(inv),
                                     _stream(stream)), "palquant_quantize_act")


def palquant_group_conv(q_dev, w_packed_dev, acc_dev, d: LayerDesc, stream=None):
    _check(lib.palquant_group_conv(_ptr(q_dev), _ptr(w_packed_dev), _ptr(acc_dev), ctypes.byref(d), _stream(stream)),
           "palquant_group_conv")


def palquant_layer_fused(q_dev, w_packed_dev, d: LayerDesc, m_out, m_req=None, shuf=None, shortcut_dev=None,
                         acc_out_dev=None, y_out_dev=None, q_out_dev=None, stream=None):
    mo = None if m_out is None else _f32(m_out)
    mr = None if m_req is None else _f32(m_req)
    _check(lib.palquant_layer_fused(_ptr(q_dev), _ptr(w_packed_dev), ctypes.byref(d), _ptr(mo), _ptr(mr),
                                    shuf or shuffle(1, 1), _ptr(shortcut_dev), _ptr(acc_out_dev), _ptr(y_out_dev),
                                    _ptr(q_out_dev), _stream(stream)), "palquant_layer_fused")


def palquant_quantize_layer_fused(x_dev, inv_s, w_packed_dev, d: LayerDesc, m_out, m_req=None, shuf=None,
                                  shortcut_dev=None, acc_out_dev=None, y_out_dev=None, q_out_dev=None, stream=None):
    inv = _f32(inv_s)
    mo = None if m_out is None else _f32(m_out)
    mr = None if m_req is None else _f32(m_req)
    _check(lib.palquant_quantize_layer_fused(_ptr(x_dev), _ptr(inv), _ptr(w_packed_dev), ctypes.byref(d), _ptr(mo),
                                             _ptr(mr), shuf or shuffle(1, 1), _ptr(shortcut_dev), _ptr(acc_out_dev),
                                             _ptr(y_out_dev), _ptr(q_out_dev), _stream(stream)),
           "palquant_quantize_layer_fused")


def palquant_cyclic_shuffle_module(q_dev, w_packed_dev, d: LayerDesc, m_out, m_req=None, shift=1, x_dev=None,
                                   z_out_dev=None, q_out_dev=None, stream=None):
    mo = None if m_out is None else _f32(m_out)
    mr = None if m_req is None else _f32(m_req)
    _check(lib.palquant_cyclic_shuffle_module(_ptr(q_dev), _ptr(w_packed_dev), ctypes.byref(d), _ptr(mo), _ptr(mr),
                                              int(shift), _ptr(x_dev), _ptr(z_out_dev), _ptr(q_out_dev),
                                              _stream(stream)), "palquant_cyclic_shuffle_module")


def palquant_sync_check(stream=None) -> int:
    return lib.palquant_sync_check(_stream(stream))


def palquant_set_wait_limit_ns(ns: int):
    _check(lib.palquant_set_wait_limit_ns(int(ns)), "palquant_set_wait_limit_ns")


def palquant_watchdog_selftest(limit_ns: int, stream=None) -> int:
    return lib.palquant_watchdog_selftest(int(limit_ns), _stream(stream))


def palquant_conv_plan(d: LayerDesc) -> ConvPlan:
    plan = ConvPlan()
    st = lib.palquant_conv_plan(ctypes.byref(d), ctypes.byref(plan))
    if st not in (PQ_OK, PQ_EUNSUPPORTED):
        raise PalquantError(st, "palquant_conv_plan")
    return plan


# Full-precision layers around the PalQuant body (first and last layers of a network).
def palquant_conv2d_f32(x_dev, w_dev, y_dev, N, H, W, Cin, Cout, k, stride, pad, relu=False, stream=None):
    _check(lib.palquant_conv2d_f32(_ptr(x_dev), _ptr(w_dev), _ptr(y_dev), N, H, W, Cin, Cout, k, stride, pad,
                                   int(bool(relu)), _stream(stream)), "palquant_conv2d_f32")


def palquant_stem_pool_f32(x_dev, w_dev, stem_dev, pool_dev, N, H, W, Cout, stream=None):
    """7x7/2 stem + ReLU and 3x3/2 max pooling in one pass; stem_dev may be None."""
    _check(lib.palquant_stem_pool_f32(_ptr(x_dev), _ptr(w_dev), _ptr(stem_dev) if stem_dev is not None else None,
                                      _ptr(pool_dev), N, H, W, Cout, _stream(stream)), "palquant_stem_pool_f32")


def palquant_maxpool2d_f32(x_dev, y_dev, N, H, W, C, k, stride, pad, stream=None):
    _check(lib.palquant_maxpool2d_f32(_ptr(x_dev), _ptr(y_dev), N, H, W, C, k, stride, pad, _stream(stream)),
           "palquant_maxpool2d_f32")


def palquant_avgpool_f32(x_dev, y_dev, N, H, W, C, stream=None):
    _check(lib.palquant_avgpool_f32(_ptr(x_dev), _ptr(y_dev), N, H, W, C, _stream(stream)), "palquant_avgpool_f32")


def palquant_linear_f32(x_dev, w_dev, y_dev, N, Cin, Cout, stream=None):
    _check(lib.palquant_linear_f32(_ptr(x_dev), _ptr(w_dev), _ptr(y_dev), N, Cin, Cout, _stream(stream)),
           "palquant_linear_f32")


# Bit-level decomposition (Eq. 4): the baseline PalQuant is compared with.
def palquant_bitsplit_desc(d: LayerDesc, bits_b: int) -> LayerDesc:
    out = LayerDesc()
    _check(lib.palquant_bitsplit_desc(ctypes.byref(d), bits_b, ctypes.byref(out)), "palquant_bitsplit_desc")
    return out


def palquant_bitsplit_scratch_bytes(d: LayerDesc, bits_b: int) -> int:
    return lib.palquant_bitsplit_scratch_bytes(ctypes.byref(d), bits_b)


def palquant_bitsplit_pack_weight_codes_host(wq_host, d: LayerDesc, bits_b: int) -> np.ndarray:
    n = palquant_packed_weight_bytes(palquant_bitsplit_desc(d, bits_b))
    out = np.empty(n, dtype=np.uint8)
    wq = np.ascontiguousarray(wq_host, dtype=np.int8)
    _check(lib.palquant_bitsplit_pack_weight_codes_host(_ptr(wq), ctypes.byref(d), bits_b, _ptr(out), n),
           "palquant_bitsplit_pack_weight_codes_host")
    return out


def palquant_bitsplit_act(q_dev, xs_dev, xs_bytes, d: LayerDesc, bits_b: int, stream=None):
    _check(lib.palquant_bitsplit_act(_ptr(q_dev), _ptr(xs_dev), xs_bytes, ctypes.byref(d), bits_b, _stream(stream)),
           "palquant_bitsplit_act")


def palquant_bitsplit_conv(q_dev, xs_dev, xs_bytes, w_packed_dev, acc_dev, d: LayerDesc, bits_b: int, stream=None):
    _check(lib.palquant_bitsplit_conv(_ptr(q_dev), _ptr(xs_dev), xs_bytes, _ptr(w_packed_dev), _ptr(acc_dev),
                                      ctypes.byref(d), bits_b, _stream(stream)), "palquant_bitsplit_conv")


def palquant_pack_weights_odd_host(w_host, d: LayerDesc, u) -> np.ndarray:
    """The paper's odd-level weight quantiser (clip range [-u, u]) and packing."""
    n = palquant_packed_weight_bytes(d)
    if n == 0:
        raise PalquantError(PQ_EUNSUPPORTED, "palquant_packed_weight_bytes")
    out = np.empty(n, dtype=np.uint8)
    w, uu = _f32(w_host), _f32(u)
    _check(lib.palquant_pack_weights_odd_host(_ptr(w), ctypes.byref(d), _ptr(uu), _ptr(out), n),
           "palquant_pack_weights_odd_host")
    return out


# ---------------------------------------------------------------- quantisation-aware training
def palquant_fake_quant_forward(x_dev, xhat_dev, P, G, Cg, bits, kind, l, u, stream=None) -> None:
    """Fake quantisation with learned per-group bounds (Eq. 2-3); kind 0 activations, 1 weights."""
    lf, uf = _f32(l), _f32(u)
    _check(lib.palquant_fake_quant_forward(_ptr(x_dev), _ptr(xhat_dev), P, G, Cg, bits, kind, _ptr(lf), _ptr(uf),
                                           _stream(stream)), "palquant_fake_quant_forward")


def palquant_fake_quant_scratch_bytes(P, G, Cg) -> int:
    return lib.palquant_fake_quant_scratch_bytes(P, G, Cg)


def palquant_fake_quant_backward(x_dev, dy_dev, dx_dev, dl_dev, du_dev, P, G, Cg, bits, kind, l, u, scratch_dev,
                                 scratch_bytes, stream=None) -> None:
    """Straight-through backward: dx (fp32) and the per-group gradients of l and u (G doubles each, device)."""
    lf, uf = _f32(l), _f32(u)
    _check(lib.palquant_fake_quant_backward(_ptr(x_dev), _ptr(dy_dev), _ptr(dx_dev), _ptr(dl_dev), _ptr(du_dev), P, G,
                                            Cg, bits, kind, _ptr(lf), _ptr(uf), _ptr(scratch_dev), scratch_bytes,
                                            _stream(stream)), "palquant_fake_quant_backward")


# ---------------------------------------------------------------- learned bounds at inference
def palquant_quantize_act_lu(x_dev, q_dev, N, H, W, G, Cg, bits, l, u, code_format=PQ_CODES_INT8, stream=None):
    """Activation codes with learned per-group bounds l < u (the training forward's codes)."""
    lf, uf = _f32(l), _f32(u)
    _check(lib.palquant_quantize_act_lu(_ptr(x_dev), _ptr(q_dev), N, H, W, G, Cg, bits, code_format, _ptr(lf),
                                        _ptr(uf), _stream(stream)), "palquant_quantize_act_lu")


def palquant_quantize_layer_fused_lu(x_dev, l, u, w_packed_dev, d: LayerDesc, m_out, m_req=None, shuf=None,
                                     shortcut_dev=None, acc_out_dev=None, y_out_dev=None, q_out_dev=None,
                                     stream=None):
    """Quantise-on-load with learned per-group bounds l < u, then the layer."""
    lf, uf = _f32(l), _f32(u)
    mo = None if m_out is None else _f32(m_out)
    mr = None if m_req is None else _f32(m_req)
    _check(lib.palquant_quantize_layer_fused_lu(_ptr(x_dev), _ptr(lf), _ptr(uf), _ptr(w_packed_dev), ctypes.byref(d),
                                                _ptr(mo), _ptr(mr), shuf or shuffle(1, 1), _ptr(shortcut_dev),
                                                _ptr(acc_out_dev), _ptr(y_out_dev), _ptr(q_out_dev), _stream(stream)),
           "palquant_quantize_layer_fused_lu")


# ---------------------------------------------------------------- 8-bit transformer layers
@functools.lru_cache(None)
def _dtypes():
    """torch's types of pq_float_type, of the token codes by code format, and of int32 sums."""
    import torch

    return ({PQ_F32: torch.float32, PQ_F16: torch.float16, PQ_BF16: torch.bfloat16},
            {PQ_CODES_INT8: torch.int8, PQ_CODES_F16: torch.float16}, torch.int32)


def _float_type(t) -> int:
    for number, dtype in _dtypes()[0].items():
        if t.dtype == dtype:
            return number
    raise TypeError(f"activations are float32, float16 or bfloat16, not {t.dtype}")


class ArgumentError(ValueError, AssertionError):
    """Tensors that a call cannot take: of other shapes, types or layouts than it was told."""


def _need(ok, message):
    if not ok:
        raise ArgumentError(message)


def _rows(t, name, columns=None):
    """Row pitch of a matrix with contiguous rows that do not overlap (any pitch for a single row)."""
    _need(t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] <= 1), f"{name}: a matrix with contiguous rows")
    _need(columns is None or t.shape[1] == columns, f"{name}: {columns} columns")
    if t.shape[0] <= 1:
        return t.shape[1]
    _need(t.stride(0) >= t.shape[1], f"{name}: rows that overlap (a pitch of {t.stride(0)} for {t.shape[1]} columns)")
    return t.stride(0)


def _layout(t):
    return t.shape, t.stride(), t.dtype, t.get_device()


_BY_HAND = object()  # a descriptor that no builder made says nothing about tensors


def _described(t, described, name):
    """Address of a call's tensor, which has the layout that its descriptor was made for (an address is the caller's word)."""
    if t is None or type(t) is int:
        return t
    if described is _BY_HAND:
        return _strided(t)
    if described is None:
        raise ArgumentError(f"{name}: not in the descriptor")
    shape, strides, dtype, device = described
    if t.shape == shape and t.dtype is dtype and t.get_device() == device and (
            t.stride() == strides or all(n <= 1 or a == b for n, a, b in zip(shape, t.stride(), strides))):
        return t.data_ptr()  # (the stride of a dimension of one element does not count)
    raise ArgumentError(f"{name}: not as the descriptor has it")


def _vector(t, dtype, count, name, device=None):
    """Address of a contiguous tensor of this type with at least `count` elements, on the device (its index) if one is known (None and
    addresses as they are)."""
    if t is None or type(t) is int:
        return t
    if t.dtype is dtype and t.numel() >= count and t.is_contiguous() and (device is None or t.get_device() == device):
        return t.data_ptr()
    raise ArgumentError(f"{name}: {count} contiguous elements of {dtype}, on the device of the other tensors")


def _room(t, nbytes, name, device=None):
    """Address of a buffer of at least `nbytes` contiguous bytes, on the device (its index) if one is known (None and addresses as they are)."""
    if t is None or type(t) is int:
        return t
    if t.is_contiguous() and t.numel() * t.element_size() >= nbytes and (device is None or t.get_device() == device):
        return t.data_ptr()
    raise ArgumentError(f"{name}: {nbytes} contiguous bytes on the device of the other tensors")


def _device_of(d, of):
    """Index of the device of the tensor that a descriptor was made for (None: filled by hand)."""
    layout = getattr(d, of, None)
    return None if layout is None else layout[3]


def _span(t, dtype, count, name, device=None):
    """Address of a tensor of this type (None: one that the library refuses) with `count` elements from its first to its last, on the
    device (its index) if one is known."""
    if t is None or type(t) is int or dtype is None:
        return _strided(t)
    if t.dtype is dtype and 1 + sum((n - 1) * step for n, step in zip(t.shape, t.stride())) >= count and (device is None or t.get_device() == device):
        return t.data_ptr()
    raise ArgumentError(f"{name}: {count} elements of {dtype}, on the device of the other tensors")


def _heads(t, name):
    """(token stride, head stride) of [tokens, heads, D] with contiguous D."""
    _need(t.dim() == 3 and (t.stride(2) == 1 or t.shape[2] <= 1), f"{name}: [tokens, heads, D] with contiguous D")
    return t.stride(0), t.stride(1)


def _heads_apart(t):
    """No element of [tokens, heads, D] lies where another does, as far as single strides tell."""
    return all(t.shape[i] <= 1 or t.stride(i) >= t.shape[2] for i in (0, 1))


def _index(t, name, count, device):
    import torch

    _need(t.dtype == torch.int32 and t.is_contiguous(), f"{name}: a contiguous int32 tensor")
    _need(t.numel() == count and t.device == device, f"{name}: {count} values, on the device of the other tensors")
    return _ptr(t)


def linear_desc(x, w, y) -> LinearDesc:
    """Descriptor of y [M, N] = x [M, K] w [N, K]^T from the tensors (w: int8 codes)."""
    import torch

    _need(w.dtype == torch.int8, "w: int8 codes")
    (M, K), N = x.shape, w.shape[0]
    _need(y.shape == (M, N), "y: [M, N]")
    _need(x.device == w.device == y.device, "x, w and y: on one device")
    d = LinearDesc(M, N, K, _float_type(x), _float_type(y), _rows(x, "x"), _rows(w, "w", K), _rows(y, "y"))
    d._x, d._w, d._y = _layout(x), _layout(w), _layout(y)
    return d


def kv8_cache(k, v, k_scale, v_scale) -> KV8Cache:
    """Descriptor of a paged 8-bit cache: codes [pages, Hkv, page_tokens, D] int8, scales [pages, Hkv] fp32.
    It keeps the tensors alive."""
    import torch

    _need(k.dim() == 4 and k.dtype == v.dtype == torch.int8 and v.shape == k.shape, "codes: two int8 tensors of one shape")
    pages, H, T, D = k.shape
    _need(k_scale.dtype == v_scale.dtype == torch.float32 and k_scale.shape == v_scale.shape == (pages, H),
          "scales: two float32 tensors [pages, Hkv]")
    _need(k.device == v.device == k_scale.device == v_scale.device, "codes and scales: on one device")
    c = KV8Cache(pages, T, H, D, _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale))
    c._keep = (k, v, k_scale, v_scale)
    c._heads, c._queries = (H, D, k.device), (D, k.device)
    return c


def kv8_tokens(k, v, cu, start, page_table, max_n) -> KV8Tokens:
    """Descriptor of the runs that k and v [tokens, Hkv, D] hold (any token and head strides; v or k may be None
    for palquant_kv8_read).  cu [B + 1], start [B], page_table [B, pages]: int32.  It keeps the index tensors alive."""
    some = k if k is not None else v
    B, dev = start.numel(), some.device
    ks, vs = ((0, 0) if t is None else _heads(t, n) for t, n in ((k, "k"), (v, "v")))
    _need(k is None or v is None or (k.shape, k.dtype, k.device) == (v.shape, v.dtype, v.device),
          "k and v: of one shape, type and device")
    _need(page_table.dim() == 2 and page_table.shape[0] == B, "page_table: [B, pages]")
    pages = page_table.shape[1]
    t = KV8Tokens(_float_type(some), B, int(max_n), pages, *ks, *vs, _index(cu, "cu", B + 1, dev),
                  _index(start, "start", B, dev), _index(page_table, "page_table", B * pages, dev))
    t._keep = (cu, start, page_table)
    t._heads = (*some.shape[1:], dev)
    t._k, t._v = (None if x is None else _layout(x) for x in (k, v))
    t._apart = all(x is None or _heads_apart(x) for x in (k, v))
    return t


def kv8_attn(q, o, cu_q, lens, page_table, max_q, max_len, scale, causal=True, window=0) -> KV8Attn:
    """Descriptor of one attention call: q and o [tokens, Hq, D] (any token and head strides), cu_q [B + 1], lens [B],
    page_table [B, pages]: int32.  It keeps the index tensors alive."""
    B, dev = lens.numel(), q.device
    q_strides, o_strides = _heads(q, "q"), _heads(o, "o")
    _need((o.shape, o.dtype, o.device) == (q.shape, q.dtype, dev), "o: as q")
    _need(_heads_apart(o), "o: outputs that overlap")
    _need(page_table.dim() == 2 and page_table.shape[0] == B, "page_table: [B, pages]")
    pages = page_table.shape[1]
    a = KV8Attn(_float_type(q), B, q.shape[1], int(max_q), int(max_len), int(bool(causal)), int(window),
                pages, float(scale), *q_strides, *o_strides, _index(cu_q, "cu_q", B + 1, dev),
                _index(lens, "lens", B, dev), _index(page_table, "page_table", B * pages, dev))
    a._keep = (cu_q, lens, page_table)
    a._queries = (q.shape[2], dev)
    a._q, a._o = _layout(q), _layout(o)
    return a


def _fits_cache(cache, d, of="_heads"):
    """A descriptor's heads, D and device against the cache's (descriptors filled by hand are not looked at)."""
    c, t = getattr(cache, of, None), getattr(d, of, None)
    if c != t and c is not None and t is not None:
        raise ArgumentError(f"{t} on a cache of {c}")


def palquant_quantize_tokens(x_dev, x_type, ldx, M, K, code_format, q_dev, ldq, s_dev, stream=None):
    """Signed 8-bit codes and one scale for each token (row); code_format PQ_CODES_INT8 or PQ_CODES_F16."""
    floats, codes, _ = _dtypes()
    at = x_dev.get_device() if getattr(x_dev, "data_ptr", None) is not None else None
    x, q, s = (_span(x_dev, floats.get(x_type), (M - 1) * ldx + K if M > 0 else 0, "x"),
               _span(q_dev, codes.get(code_format), (M - 1) * ldq + K if M > 0 else 0, "q", at),
               _vector(s_dev, floats[PQ_F32], M, "s", at))
    _check(lib.palquant_quantize_tokens(x, x_type, ldx, M, K, code_format, q, ldq, s, _stream(stream)),
           "palquant_quantize_tokens")


def palquant_linear_code_format(d: LinearDesc) -> int:
    return lib.palquant_linear_code_format(ctypes.byref(d))


def palquant_linear_i8(q_dev, code_format, ldq, s_x_dev, w_dev, s_w_dev, bias_dev, acc_dev, y_dev, d: LinearDesc,
                       stream=None):
    """Dense layer on token codes: exact int32 sums, scales for each token and output channel."""
    floats, codes, sums = _dtypes()
    M, N, f32, at = d.M, d.N, floats[PQ_F32], _device_of(d, "_w")
    q = _span(q_dev, codes.get(code_format), (M - 1) * ldq + d.K if M > 0 else 0, "q", at)
    _check(lib.palquant_linear_i8(q, code_format, ldq, _vector(s_x_dev, f32, M, "s_x", at), _described(w_dev, getattr(d, "_w", _BY_HAND), "w"),
                                  _vector(s_w_dev, f32, N, "s_w", at), _vector(bias_dev, f32, N, "bias", at),
                                  _vector(acc_dev, sums, M * N, "acc", at), _described(y_dev, getattr(d, "_y", _BY_HAND), "y"),
                                  ctypes.byref(d), _stream(stream)), "palquant_linear_i8")


def palquant_linear_q8_scratch_bytes(d: LinearDesc) -> int:
    return lib.palquant_linear_q8_scratch_bytes(ctypes.byref(d))


def palquant_linear_q8(x_dev, w_dev, s_w_dev, bias_dev, y_dev, d: LinearDesc, scratch_dev, scratch_bytes, stream=None):
    """Token quantiser and dense layer: x to y."""
    N, f32, at = d.N, _dtypes()[0][PQ_F32], _device_of(d, "_x")
    _check(lib.palquant_linear_q8(_described(x_dev, getattr(d, "_x", _BY_HAND), "x"), _described(w_dev, getattr(d, "_w", _BY_HAND), "w"),
                                  _vector(s_w_dev, f32, N, "s_w", at), _vector(bias_dev, f32, N, "bias", at),
                                  _described(y_dev, getattr(d, "_y", _BY_HAND), "y"), ctypes.byref(d),
                                  _room(scratch_dev, scratch_bytes, "scratch", at), scratch_bytes, _stream(stream)), "palquant_linear_q8")


def palquant_kv8_append(cache: KV8Cache, k_dev, v_dev, t: KV8Tokens, stream=None):
    """Quantise runs of tokens into the cache (one scale for each page and head)."""
    _fits_cache(cache, t)
    _check(lib.palquant_kv8_append(ctypes.byref(cache), _described(k_dev, getattr(t, "_k", _BY_HAND), "k"),
                                   _described(v_dev, getattr(t, "_v", _BY_HAND), "v"), ctypes.byref(t), _stream(stream)),
           "palquant_kv8_append")


def palquant_kv8_read(cache: KV8Cache, k_dev, v_dev, t: KV8Tokens, stream=None):
    """The values that runs of cached tokens stand for; k_dev or v_dev may be None."""
    _fits_cache(cache, t)
    _need(getattr(t, "_apart", True), "k, v: outputs that overlap")
    _check(lib.palquant_kv8_read(ctypes.byref(cache), _described(k_dev, getattr(t, "_k", _BY_HAND), "k"),
                                 _described(v_dev, getattr(t, "_v", _BY_HAND), "v"), ctypes.byref(t), _stream(stream)),
           "palquant_kv8_read")


def palquant_kv8_attention_scratch_bytes(cache: KV8Cache, a: KV8Attn) -> int:
    return lib.palquant_kv8_attention_scratch_bytes(ctypes.byref(cache), ctypes.byref(a))


def palquant_kv8_attention(cache: KV8Cache, q_dev, o_dev, a: KV8Attn, scratch_dev, scratch_bytes, stream=None):
    """Attention over the cache: single tokens, chunks and prompts, grouped heads."""
    _fits_cache(cache, a, "_queries")
    _check(lib.palquant_kv8_attention(ctypes.byref(cache), _described(q_dev, getattr(a, "_q", _BY_HAND), "q"),
                                      _described(o_dev, getattr(a, "_o", _BY_HAND), "o"), ctypes.byref(a),
                                      _room(scratch_dev, scratch_bytes, "scratch", _device_of(a, "_q")), scratch_bytes, _stream(stream)),
           "palquant_kv8_attention")


# ---------------------------------------------------------------- a decoder's operators around the 8-bit cache
_get_device = None  # torch's function for the current device


def _here(device):
    """A call's tensors lie on the current device (its index), whose stream the call takes."""
    global _get_device
    if device is None:
        return  # a descriptor that no builder made, or addresses: the caller's word
    if _get_device is None:
        import torch

        _get_device = torch._C._cuda_getDevice
    if device < 0 or device != _get_device():
        raise ArgumentError(f"tensors on {'the CPU' if device < 0 else f'cuda:{device}'}: not the current device")


def _index_of(t):
    return None if t is None or type(t) is int else t.get_device()


def _same_or_apart(src, dst, name):
    """An output that starts where its input does is the input itself."""
    _need(dst.data_ptr() != src.data_ptr() or _layout(dst) == _layout(src) or not dst.numel(),
          f"{name}: the input itself, or elsewhere")


def rope_turns(frequencies, device):
    """The rotation's frequencies (radians a position, one for each pair of elements) as palquant_qk_norm_rope reads them."""
    import torch

    f = np.ascontiguousarray(np.asarray(frequencies, dtype=np.float64))
    _need(f.ndim == 1, "frequencies: one for each pair")
    turns = np.empty(f.shape, np.uint64)
    _check(lib.palquant_rope_turns_host(_ptr(f), f.size, _ptr(turns)), "palquant_rope_turns_host")
    return torch.from_numpy(turns.view(np.int64)).to(device)


def qk_norm_rope(q, k, q_out, k_out, positions=None, turns=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                 norm=True) -> QKRope:
    """Descriptor of a call on queries and keys [tokens, heads, D] (any token and head strides; one of them may be None, with its
    output): norms with a weight for each element (None: ones; norm=False: no norm), rotation of the first 2 * len(turns)
    elements by positions [tokens] (int32; turns=None: no rotation).  An output is its input itself or apart from the
    inputs and the other output.  It keeps positions, turns and weights alive."""
    import torch

    some = q if q is not None else k
    _need(some is not None and (q is None) == (q_out is None) and (k is None) == (k_out is None), "q, k: at least one, with its output")
    tokens, D, dev = some.shape[0], some.shape[-1], some.device
    strides, heads = [], []
    for name, x, y in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            strides.append((0, 0, 0, 0))
            heads.append(0)
            continue
        strides.append(_heads(x, name) + _heads(y, name + "_out"))
        _need(x.shape[0] == tokens and x.shape[2] == D and (x.dtype, x.device) == (some.dtype, dev), "q and k: of one length, D, type and device")
        _need((y.shape, y.dtype, y.device) == (x.shape, x.dtype, dev), f"{name}_out: as {name}")
        _need(_heads_apart(y), f"{name}_out: outputs that overlap")
        _same_or_apart(x, y, name + "_out")
        heads.append(x.shape[1])
    w_type, keep = PQ_F32, []
    _need(norm or (q_weight is None and k_weight is None), "weights: of a norm")
    weights = [w for w in (q_weight, k_weight) if w is not None]
    if weights:
        w_type = _float_type(weights[0])
        for w in weights:
            _need(w.dtype == weights[0].dtype and w.shape == (D,) and w.is_contiguous() and w.device == dev, "weights: [D] of one type")
    R = 0
    if turns is not None:
        _need(turns.dtype == torch.int64 and turns.dim() == 1 and turns.is_contiguous() and turns.device == dev, "turns: those of rope_turns")
        R = 2 * turns.numel()
        _need(R <= D, "turns: one for each pair of elements at most")
        _need(positions is not None, "positions: one for each token")
        keep += [turns, positions]
    d = QKRope(_float_type(some), w_type, tokens, *heads, D, R, int(bool(interleaved)), int(bool(norm)), float(eps), *strides[0][:2],
               *strides[1][:2], *strides[0][2:], *strides[1][2:], _index(positions, "positions", tokens, dev) if R else None,
               _ptr(turns) if R else None, _ptr(q_weight), _ptr(k_weight))
    d._keep = keep + weights
    d._q, d._k, d._q_out, d._k_out = (None if x is None else _layout(x) for x in (q, k, q_out, k_out))
    d._device = some.get_device()
    return d


def palquant_qk_norm_rope(q_dev, k_dev, q_out_dev, k_out_dev, d: QKRope, stream=None):
    """Norms of query and key heads and the rotation by position, in one pass."""
    _here(getattr(d, "_device", None))
    layouts = [getattr(d, name, _BY_HAND) for name in ("_q", "_k", "_q_out", "_k_out")]
    q, k = _described(q_dev, layouts[0], "q"), _described(k_dev, layouts[1], "k")
    q_out, k_out = _described(q_out_dev, layouts[2], "q_out"), _described(k_out_dev, layouts[3], "k_out")
    # an output that starts where its input does is the input itself
    _need((q is None or q != q_out or layouts[0] == layouts[2]) and (k is None or k != k_out or layouts[1] == layouts[3]),
          "q_out, k_out: the input itself, or elsewhere")
    _check(lib.palquant_qk_norm_rope(q, k, q_out, k_out, ctypes.byref(d), _stream(stream)), "palquant_qk_norm_rope")


def w4_weights(N, K, group, scales) -> W4Weights:
    """Descriptor of packed 4-bit weights [N, K] with a scale (of torch type `scales`) for each channel and `group` of K."""
    types = {dtype: number for number, dtype in _dtypes()[0].items()}
    _need(scales in types, "scales: float32, float16 or bfloat16")
    w = W4Weights(N, K, group, types[scales])
    w._bytes = lib.palquant_w4_packed_bytes(ctypes.byref(w))
    return w


def palquant_w4_packed_bytes(w: W4Weights) -> int:
    return lib.palquant_w4_packed_bytes(ctypes.byref(w))


def palquant_w4_pack(codes_dev, s_dev, w: W4Weights, packed_dev, packed_bytes, stream=None):
    """Codes [N, K] (int8, -8 to 7) and scales [N, groups] into the layout of the products."""
    import torch

    ldc = w.K
    at = _index_of(packed_dev)
    _here(at)
    _need(at is None or all(_index_of(t) in (None, at) for t in (codes_dev, s_dev)), "codes and scales: on the device of packed")
    if getattr(codes_dev, "data_ptr", None) is not None:
        _need(codes_dev.dtype == torch.int8 and codes_dev.shape == (w.N, w.K), "codes: int8 [N, K]")
        ldc = _rows(codes_dev, "codes")
    groups = -(-w.K // w.group) if w.group > 0 else 0
    _check(lib.palquant_w4_pack(_strided(codes_dev), ldc, _vector(s_dev, _dtypes()[0].get(w.s_type), w.N * groups, "scales"), ctypes.byref(w),
                                _room(packed_dev, packed_bytes, "packed"), packed_bytes, _stream(stream)), "palquant_w4_pack")


def palquant_w4_quantize(w_dev, w_type, ldw, w: W4Weights, packed_dev, packed_bytes, stream=None):
    """Float weights [N, K] (rows `ldw` elements apart) quantised to 4 bits and packed."""
    at = _index_of(packed_dev)
    _here(at)
    _need(at is None or _index_of(w_dev) in (None, at), "w: on the device of packed")
    _check(lib.palquant_w4_quantize(_span(w_dev, _dtypes()[0].get(w_type), (w.N - 1) * ldw + w.K, "w"), w_type, ldw, ctypes.byref(w),
                                    _room(packed_dev, packed_bytes, "packed"), packed_bytes, _stream(stream)), "palquant_w4_quantize")


def palquant_w4_unpack(packed_dev, w: W4Weights, codes_dev, s_dev, stream=None):
    """The codes (int8 [N, K]) and fp32 scales [N, groups] that packed weights hold; either may be None."""
    import torch

    ldc = w.K
    at = _index_of(packed_dev)
    _here(at)
    _need(at is None or all(_index_of(t) in (None, at) for t in (codes_dev, s_dev)), "codes and scales: on the device of packed")
    if getattr(codes_dev, "data_ptr", None) is not None:
        _need(codes_dev.dtype == torch.int8 and codes_dev.shape == (w.N, w.K), "codes: int8 [N, K]")
        ldc = _rows(codes_dev, "codes")
    groups = -(-w.K // w.group) if w.group > 0 else 0
    _check(lib.palquant_w4_unpack(_room(packed_dev, palquant_w4_packed_bytes(w), "packed"), ctypes.byref(w), _strided(codes_dev), ldc,
                                  _vector(s_dev, _dtypes()[0][PQ_F32], w.N * groups, "scales"), _stream(stream)), "palquant_w4_unpack")


def linear_w4_desc(x, w: W4Weights, y) -> LinearDesc:
    """Descriptor of y [M, N] = x [M, K] times packed 4-bit weights."""
    M = x.shape[0]
    _need(x.dim() == 2 and x.shape[1] == w.K and y.shape == (M, w.N), "x: [M, K], y: [M, N]")
    _need(x.device == y.device, "x and y: on one device")
    d = LinearDesc(M, w.N, w.K, _float_type(x), _float_type(y), _rows(x, "x"), w.K, _rows(y, "y"))
    d._x, d._y, d._device = _layout(x), _layout(y), x.get_device()
    return d


def palquant_linear_w4_scratch_bytes(w: W4Weights, d: LinearDesc) -> int:
    return lib.palquant_linear_w4_scratch_bytes(ctypes.byref(w), ctypes.byref(d))


def palquant_linear_w4(x_dev, packed_dev, bias_dev, y_dev, w: W4Weights, d: LinearDesc, scratch_dev, scratch_bytes, stream=None):
    """Dense layer with 4-bit weights and group scales: x to y."""
    at = getattr(d, "_device", None)
    _here(at)
    nbytes = getattr(w, "_bytes", None)
    if nbytes is None:
        nbytes = lib.palquant_w4_packed_bytes(ctypes.byref(w))
    packed = _room(packed_dev, nbytes, "packed", at)
    _check(lib.palquant_linear_w4(_described(x_dev, getattr(d, "_x", _BY_HAND), "x"), packed, _vector(bias_dev, _dtypes()[0][PQ_F32], d.N, "bias", at),
                                  _described(y_dev, getattr(d, "_y", _BY_HAND), "y"), ctypes.byref(w), ctypes.byref(d),
                                  _room(scratch_dev, scratch_bytes, "scratch", at), scratch_bytes, _stream(stream)), "palquant_linear_w4")


def palquant_kv8_attention_sinks_scratch_bytes(cache: KV8Cache, a: KV8Attn, sinks) -> int:
    return lib.palquant_kv8_attention_sinks_scratch_bytes(ctypes.byref(cache), ctypes.byref(a), sinks)


def palquant_kv8_attention_sinks(cache: KV8Cache, q_dev, o_dev, a: KV8Attn, sinks, scratch_dev, scratch_bytes, stream=None):
    """Attention over the cache through a window, with the first `sinks` tokens of every sequence in sight."""
    at = _device_of(a, "_q")
    _here(at)
    _fits_cache(cache, a, "_queries")
    _check(lib.palquant_kv8_attention_sinks(ctypes.byref(cache), _described(q_dev, getattr(a, "_q", _BY_HAND), "q"),
                                            _described(o_dev, getattr(a, "_o", _BY_HAND), "o"), ctypes.byref(a), sinks,
                                            _room(scratch_dev, scratch_bytes, "scratch", at), scratch_bytes, _stream(stream)),
           "palquant_kv8_attention_sinks")


def kv8_tree(bits, a: KV8Attn) -> KV8Tree:
    """Descriptor of which drafts each draft sees: bits [tokens, words] (int32, contiguous rows), a row for each of a's
    queries, bit j % 32 of word j / 32 for the sequence's draft j.  It keeps the bits alive."""
    import torch

    _need(bits.dtype == torch.int32, "bits: int32")
    pitch = _rows(bits, "bits")
    q = getattr(a, "_q", None)
    _need(q is None or (bits.shape[0] == q[0][0] and bits.get_device() == q[3]), "bits: a row for each query, on its device")
    t = KV8Tree(_strided(bits), pitch, bits.shape[1])
    t._keep, t._for = bits, q
    return t


def palquant_kv8_attention_tree_scratch_bytes(cache: KV8Cache, a: KV8Attn, tree: KV8Tree) -> int:
    return lib.palquant_kv8_attention_tree_scratch_bytes(ctypes.byref(cache), ctypes.byref(a), ctypes.byref(tree))


def palquant_kv8_attention_tree(cache: KV8Cache, q_dev, o_dev, a: KV8Attn, tree: KV8Tree, scratch_dev, scratch_bytes, stream=None):
    """Attention for drafted tokens, the sequences' last cached ones: each sees the text before them and the drafts of its bits."""
    at = _device_of(a, "_q")
    _here(at)
    _fits_cache(cache, a, "_queries")
    _need(getattr(tree, "_for", None) == getattr(a, "_q", None) or not hasattr(tree, "_for"), "tree: of other queries")
    _check(lib.palquant_kv8_attention_tree(ctypes.byref(cache), _described(q_dev, getattr(a, "_q", _BY_HAND), "q"),
                                           _described(o_dev, getattr(a, "_o", _BY_HAND), "o"), ctypes.byref(a), ctypes.byref(tree),
                                           _room(scratch_dev, scratch_bytes, "scratch", at), scratch_bytes, _stream(stream)),
           "palquant_kv8_attention_tree")
