"""Python binding of libsamd (argument marshalling only).

The functions named like the C ABI (samd_pack, samd_conv2d, ...) take torch
CUDA tensors, pass their device pointers and the current CUDA stream to the
library, and raise SamdError on a non-zero status. Every step of the
computation runs in libsamd's CUDA kernels; nothing here computes a result.
The helpers without the prefix (pack, conv2d, ...) only allocate the output
tensors with torch and call those bindings.

If libsamd.so is missing and cannot be built, load() raises: there is no
fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import struct
from dataclasses import dataclass

import torch

from . import build as _build

# ---- C types -----------------------------------------------------------------


class samd_fmt(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_uint8), ("is_signed", ctypes.c_uint8), ("spacer", ctypes.c_uint8),
                ("word_bits", ctypes.c_uint8)]

    def __repr__(self):
        return f"samd_fmt(bits={self.bits}, is_signed={self.is_signed}, spacer={self.spacer}, word_bits={self.word_bits})"


class samd_conv_desc(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int), ("C", ctypes.c_int), ("H", ctypes.c_int), ("W", ctypes.c_int),
                ("K", ctypes.c_int), ("R", ctypes.c_int), ("S", ctypes.c_int), ("stride", ctypes.c_int),
                ("pad", ctypes.c_int), ("layout", ctypes.c_int)]


class samd_matvec_desc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int), ("N", ctypes.c_int), ("K", ctypes.c_int), ("group", ctypes.c_int),
                ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64), ("type", ctypes.c_int)]


class samd_weights4(ctypes.Structure):
    _fields_ = [("lanes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("zeros", ctypes.c_void_p)]


class samd_block8(ctypes.Structure):
    _fields_ = [("lanes", ctypes.c_void_p), ("exps", ctypes.c_void_p)]


class samd_ffn_desc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int), ("K", ctypes.c_int), ("F", ctypes.c_int), ("ldx", ctypes.c_int64),
                ("ldw", ctypes.c_int64), ("ldh", ctypes.c_int64), ("type", ctypes.c_int), ("act", ctypes.c_int)]


class samd_cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int), ("page", ctypes.c_int), ("heads", ctypes.c_int), ("dim", ctypes.c_int),
                ("fmt", samd_fmt), ("type", ctypes.c_int), ("k_lanes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p),
                ("v_lanes", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class samd_cache_seqs(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int), ("max_pages", ctypes.c_int), ("ld", ctypes.c_int64), ("table", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p)]


class samd_moe_desc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int), ("K", ctypes.c_int), ("F", ctypes.c_int), ("E", ctypes.c_int), ("topk", ctypes.c_int),
                ("group", ctypes.c_int), ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64), ("type", ctypes.c_int),
                ("act", ctypes.c_int)]


SAMD_OK, SAMD_EINVAL, SAMD_EALIGN, SAMD_ESHAPE, SAMD_EUNSUP, SAMD_ECUDA, SAMD_ETIMEOUT = range(7)
SAMD_ADD, SAMD_SUB, SAMD_MUL, SAMD_RELU, SAMD_REQUANT = range(5)
SAMD_NCHW, SAMD_NHWC = 0, 1
SAMD_F16, SAMD_BF16, SAMD_F32 = range(3)
DTYPES = {torch.float16: SAMD_F16, torch.bfloat16: SAMD_BF16, torch.float32: SAMD_F32}
SAMD_SILU, SAMD_GELU, SAMD_GELU_TANH, SAMD_RELU_ACT = range(4)
ACTS = {"silu": SAMD_SILU, "gelu": SAMD_GELU, "gelu_tanh": SAMD_GELU_TANH, "relu": SAMD_RELU_ACT}
OPS = {"add": SAMD_ADD, "sub": SAMD_SUB, "mul": SAMD_MUL, "relu": SAMD_RELU, "requant": SAMD_REQUANT}

EXPORTED = ["samd_lanes_per_word", "samd_packed_words", "samd_pack", "samd_unpack", "samd_elementwise",
            "samd_conv2d", "samd_conv2d_workspace_size", "samd_conv2d_operand_bits", "samd_conv2d_set_min_tiles_per_cta", "samd_conv2d_prepare", "samd_conv2d_prepared",
            "samd_conv2d_noalloc", "samd_conv2d_prepared_pool2x2", "samd_conv2d_pool2x2_supported",
            "samd_matvec4", "samd_gated_matvec4", "samd_block8_quantize", "samd_block8_dequantize",
            "samd_gated_ffn_forward", "samd_gated_ffn_backward", "samd_gated_ffn_backward_workspace_size",
            "samd_cache_append", "samd_cache_read", "samd_paged_attention", "samd_paged_attention_workspace_size",
            "samd_cache_evict", "samd_moe_route", "samd_moe4", "samd_moe4_workspace_size",
            "samd_maxpool2x2", "samd_device_status", "samd_selftest_wait_timeout", "samd_status_str", "samd_version"]
FMT_NONE = (0, 0, 0, 0)


class SamdError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_str(status)}")


_lib = None


def lib_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True):
    """Load libsamd.so (building it in-tree first if it is missing or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing and not _build.up_to_date():
        _build.build()
    if not os.path.exists(_build.LIB):
        raise RuntimeError(f"libsamd.so not found at {_build.LIB}; the CUDA path has no fallback")
    lib = ctypes.CDLL(_build.LIB)
    c = ctypes
    vp, i64, i32, sz = c.c_void_p, c.c_int64, c.c_int, c.c_size_t
    lib.samd_lanes_per_word.argtypes, lib.samd_lanes_per_word.restype = [samd_fmt], sz
    lib.samd_packed_words.argtypes, lib.samd_packed_words.restype = [samd_fmt, i64, i64], i64
    lib.samd_pack.argtypes, lib.samd_pack.restype = [samd_fmt, vp, vp, i64, i64, vp], i32
    lib.samd_unpack.argtypes, lib.samd_unpack.restype = [samd_fmt, vp, vp, i64, i64, vp], i32
    lib.samd_elementwise.argtypes = [i32, samd_fmt, vp, vp, samd_fmt, vp, i64, i32, i32, vp]
    lib.samd_elementwise.restype = i32
    lib.samd_conv2d.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, vp, samd_fmt, vp, vp, samd_fmt, vp, i32, vp, sz,
                                vp]
    lib.samd_conv2d.restype = i32
    lib.samd_conv2d_noalloc.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, vp, samd_fmt, vp, vp, samd_fmt, vp, i32,
                                        vp]
    lib.samd_conv2d_noalloc.restype = i32
    lib.samd_conv2d_prepare.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, samd_fmt, vp, samd_fmt, vp, sz, vp]
    lib.samd_conv2d_prepare.restype = i32
    lib.samd_conv2d_prepared.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, vp, samd_fmt, vp, sz, vp, samd_fmt, vp,
                                         i32, vp]
    lib.samd_conv2d_prepared.restype = i32
    lib.samd_conv2d_prepared_pool2x2.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, vp, samd_fmt, vp, sz, samd_fmt,
                                                 vp, i32, vp]
    lib.samd_conv2d_prepared_pool2x2.restype = i32
    lib.samd_conv2d_pool2x2_supported.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, samd_fmt, samd_fmt]
    lib.samd_conv2d_pool2x2_supported.restype = i32
    lib.samd_conv2d_workspace_size.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, samd_fmt]
    lib.samd_conv2d_workspace_size.restype = sz
    lib.samd_conv2d_operand_bits.argtypes = [c.POINTER(samd_conv_desc), samd_fmt, samd_fmt]
    lib.samd_conv2d_operand_bits.restype = i32
    lib.samd_conv2d_set_min_tiles_per_cta.argtypes = [i32]
    lib.samd_conv2d_set_min_tiles_per_cta.restype = i32
    lib.samd_maxpool2x2.argtypes = [samd_fmt, vp, vp, i32, i32, i32, i32, i32, vp]
    lib.samd_maxpool2x2.restype = i32
    mvp, w4, b8, fdp = c.POINTER(samd_matvec_desc), samd_weights4, samd_block8, c.POINTER(samd_ffn_desc)
    lib.samd_matvec4.argtypes, lib.samd_matvec4.restype = [mvp, samd_fmt, vp, w4, vp, vp], i32
    lib.samd_gated_matvec4.argtypes = [mvp, i32, samd_fmt, vp, w4, w4, vp, vp]
    lib.samd_gated_matvec4.restype = i32
    lib.samd_block8_quantize.argtypes, lib.samd_block8_quantize.restype = [i32, vp, i64, i64, i64, b8, vp], i32
    lib.samd_block8_dequantize.argtypes, lib.samd_block8_dequantize.restype = [i32, b8, i64, i64, vp, i64, vp], i32
    lib.samd_gated_ffn_forward.argtypes = [fdp, vp, vp, vp, vp, b8, b8, vp]
    lib.samd_gated_ffn_forward.restype = i32
    lib.samd_gated_ffn_backward.argtypes = [fdp, vp, b8, b8, b8, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.samd_gated_ffn_backward.restype = i32
    lib.samd_gated_ffn_backward_workspace_size.argtypes = [fdp]
    lib.samd_gated_ffn_backward_workspace_size.restype = sz
    cp, sp, f32 = c.POINTER(samd_cache), c.POINTER(samd_cache_seqs), c.c_float
    lib.samd_cache_append.argtypes, lib.samd_cache_append.restype = [cp, sp, vp, i32, vp, i64, vp, i64, vp], i32
    lib.samd_cache_read.argtypes, lib.samd_cache_read.restype = [cp, sp, vp, i32, vp, i64, vp, i64, vp], i32
    lib.samd_paged_attention.argtypes = [cp, sp, i32, vp, i64, f32, vp, i64, vp, i64, vp, sz, vp]
    lib.samd_paged_attention.restype = i32
    lib.samd_paged_attention_workspace_size.argtypes = [cp, sp, i32, i32]
    lib.samd_paged_attention_workspace_size.restype = sz
    lib.samd_cache_evict.argtypes = [cp, sp, vp, i64, i32, i32, vp, i64, vp, vp, vp, vp]
    lib.samd_cache_evict.restype = i32
    xdp = c.POINTER(samd_moe_desc)
    lib.samd_moe_route.argtypes, lib.samd_moe_route.restype = [xdp, i32, vp, vp, vp, vp, vp], i32
    lib.samd_moe4.argtypes, lib.samd_moe4.restype = [xdp, samd_fmt, vp, vp, vp, w4, w4, w4, vp, vp, sz, vp], i32
    lib.samd_moe4_workspace_size.argtypes, lib.samd_moe4_workspace_size.restype = [xdp], sz
    lib.samd_device_status.argtypes, lib.samd_device_status.restype = [c.POINTER(c.c_int), i32, vp], i32
    lib.samd_selftest_wait_timeout.argtypes, lib.samd_selftest_wait_timeout.restype = [c.c_uint64, vp], i32
    lib.samd_status_str.argtypes, lib.samd_status_str.restype = [i32], c.c_char_p
    lib.samd_version.argtypes, lib.samd_version.restype = [], c.c_char_p
    _lib = lib
    return lib


def status_str(status: int) -> str:
    return load().samd_status_str(status).decode()


def _check(status: int, what: str) -> None:
    if status != SAMD_OK:
        raise SamdError(status, what)


def _ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        return t  # an integer address
    if not t.is_cuda:
        raise ValueError("libsamd takes device tensors")
    return t.data_ptr()


# The raw handle of the current stream of a device: what current_stream().cuda_stream is, without an object in
# between (3 us a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ---- formats -------------------------------------------------------------------


def fmt(bits: int, signed: bool, spacer: int = 0, word_bits: int = 32) -> samd_fmt:
    return samd_fmt(bits, int(bool(signed)), spacer, word_bits)


def word_dtype(f: samd_fmt) -> torch.dtype:
    """torch dtype that stores one packed word (bit pattern)."""
    return torch.int32 if f.word_bits == 32 else torch.int64


def samd_lanes_per_word(f: samd_fmt) -> int:
    return int(load().samd_lanes_per_word(f))


def samd_packed_words(f: samd_fmt, rows: int, inner: int) -> int:
    return int(load().samd_packed_words(f, rows, inner))


# ---- the C ABI, one binding per entry point -------------------------------------


def samd_pack(f, src, dst, rows, inner, stream=None):
    _check(load().samd_pack(f, _ptr(src), _ptr(dst), rows, inner, _stream(stream)), "samd_pack")


def samd_unpack(f, src, dst, rows, inner, stream=None):
    _check(load().samd_unpack(f, _ptr(src), _ptr(dst), rows, inner, _stream(stream)), "samd_unpack")


def samd_elementwise(op, fa, a, b, fo, out, n, shift=0, saturate=0, stream=None):
    op = OPS[op] if isinstance(op, str) else op
    _check(load().samd_elementwise(op, fa, _ptr(a), _ptr(b), fo, _ptr(out), n, shift, int(saturate),
                                   _stream(stream)), "samd_elementwise")


def samd_conv2d_workspace_size(desc: samd_conv_desc, fa: samd_fmt, fw: samd_fmt) -> int:
    return int(load().samd_conv2d_workspace_size(ctypes.byref(desc), fa, fw))


def samd_conv2d_set_min_tiles_per_cta(tiles: int) -> None:
    """Minimum 128-pixel tiles per SM of a convolution launch (1: spread each layer
    over every SM; larger: leave SMs to layers running on other streams)."""
    _check(load().samd_conv2d_set_min_tiles_per_cta(int(tiles)), "samd_conv2d_set_min_tiles_per_cta")


def samd_conv2d_operand_bits(desc: samd_conv_desc, fa: samd_fmt, fw: samd_fmt) -> int:
    """8 (e4m3) or 16 (fp16): the tensor-core operand type of this convolution; 0 if rejected."""
    return int(load().samd_conv2d_operand_bits(ctypes.byref(desc), fa, fw))


def samd_conv2d(desc, fa, act, fw, wt, acc_out, fo, packed_out, shift, workspace, workspace_bytes=None,
                stream=None):
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size() if isinstance(workspace, torch.Tensor) else 0
    _check(load().samd_conv2d(ctypes.byref(desc), fa, _ptr(act), fw, _ptr(wt), _ptr(acc_out),
                              fo if fo is not None else samd_fmt(8, 1, 0, 32), _ptr(packed_out), shift,
                              _ptr(workspace), workspace_bytes, _stream(stream)), "samd_conv2d")


def samd_conv2d_noalloc(desc, fa, act, fw, wt, acc_out, fo, packed_out, shift, stream=None):
    """samd_conv2d without a workspace (the library's static scratch holds the widened weights)."""
    _check(load().samd_conv2d_noalloc(ctypes.byref(desc), fa, _ptr(act), fw, _ptr(wt), _ptr(acc_out),
                                      fo if fo is not None else samd_fmt(8, 1, 0, 32), _ptr(packed_out), shift,
                                      _stream(stream)), "samd_conv2d_noalloc")


def _nbytes(t):
    return t.numel() * t.element_size() if isinstance(t, torch.Tensor) else 0


def samd_conv2d_prepare(desc, fa, fw, wt, fo, prepared, prepared_bytes=None, stream=None):
    fo = fo if fo is not None else samd_fmt(*FMT_NONE)
    nb = _nbytes(prepared) if prepared_bytes is None else prepared_bytes
    _check(load().samd_conv2d_prepare(ctypes.byref(desc), fa, fw, _ptr(wt), fo, _ptr(prepared), nb, _stream(stream)),
           "samd_conv2d_prepare")


def samd_conv2d_prepared(desc, fa, act, fw, prepared, acc_out, fo, packed_out, shift, prepared_bytes=None,
                         stream=None):
    fo = fo if fo is not None else samd_fmt(*FMT_NONE)
    nb = _nbytes(prepared) if prepared_bytes is None else prepared_bytes
    _check(load().samd_conv2d_prepared(ctypes.byref(desc), fa, _ptr(act), fw, _ptr(prepared), nb, _ptr(acc_out), fo,
                                       _ptr(packed_out), shift, _stream(stream)), "samd_conv2d_prepared")


def samd_conv2d_prepared_pool2x2(desc, fa, act, fw, prepared, fo, pooled_out, shift, prepared_bytes=None,
                                 stream=None):
    nb = _nbytes(prepared) if prepared_bytes is None else prepared_bytes
    _check(load().samd_conv2d_prepared_pool2x2(ctypes.byref(desc), fa, _ptr(act), fw, _ptr(prepared), nb, fo,
                                               _ptr(pooled_out), shift, _stream(stream)),
           "samd_conv2d_prepared_pool2x2")


def samd_conv2d_pool2x2_supported(desc, fa, fw, fo) -> bool:
    return bool(load().samd_conv2d_pool2x2_supported(ctypes.byref(desc), fa, fw, fo))


def samd_maxpool2x2(f, inp, out, N, C, H, W, layout=SAMD_NHWC, stream=None):
    _check(load().samd_maxpool2x2(f, _ptr(inp), _ptr(out), N, C, H, W, layout, _stream(stream)),
           "samd_maxpool2x2")


def _weights4(lanes, scales, zeros) -> samd_weights4:
    return samd_weights4(_ptr(lanes), _ptr(scales), _ptr(zeros))


def _block8(b) -> samd_block8:
    """Of a Block8, a pair (lanes, exps) of tensors or addresses, or None."""
    if b is None:
        return samd_block8(None, None)
    if isinstance(b, Block8) and b._buf is not None:
        p = _ptr(b._buf)
        return samd_block8(p, p + 4 * b._lane_words())
    return samd_block8(_ptr(b[0]), _ptr(b[1]))


def _act(act) -> int:
    return ACTS[act] if isinstance(act, str) else act


def samd_matvec4(desc: samd_matvec_desc, fw, x, lanes, scales, zeros, y, stream=None):
    _check(load().samd_matvec4(ctypes.byref(desc), fw, _ptr(x), _weights4(lanes, scales, zeros), _ptr(y),
                               _stream(stream)), "samd_matvec4")


def samd_gated_matvec4(desc: samd_matvec_desc, act, fw, x, wg, wu, y, stream=None):
    """wg, wu: (lanes, scales, zeros or None)."""
    _check(load().samd_gated_matvec4(ctypes.byref(desc), _act(act), fw, _ptr(x), _weights4(*wg), _weights4(*wu),
                                     _ptr(y), _stream(stream)), "samd_gated_matvec4")


def samd_block8_quantize(dtype, x, ldx, rows, inner, out, stream=None):
    _check(load().samd_block8_quantize(DTYPES.get(dtype, dtype), _ptr(x), ldx, rows, inner, _block8(out),
                                       _stream(stream)), "samd_block8_quantize")


def samd_block8_dequantize(dtype, b, rows, inner, y, ldy, stream=None):
    _check(load().samd_block8_dequantize(DTYPES.get(dtype, dtype), _block8(b), rows, inner, _ptr(y), ldy,
                                         _stream(stream)), "samd_block8_dequantize")


def samd_gated_ffn_forward(desc: samd_ffn_desc, x, wg, wu, h, ckpt_g=None, ckpt_u=None, stream=None):
    _check(load().samd_gated_ffn_forward(ctypes.byref(desc), _ptr(x), _ptr(wg), _ptr(wu), _ptr(h), _block8(ckpt_g),
                                         _block8(ckpt_u), _stream(stream)), "samd_gated_ffn_forward")


def samd_gated_ffn_backward_workspace_size(desc: samd_ffn_desc) -> int:
    return int(load().samd_gated_ffn_backward_workspace_size(ctypes.byref(desc)))


def samd_gated_ffn_backward(desc: samd_ffn_desc, dh, ckpt_x, ckpt_g, ckpt_u, wg, wu, dx, dwg, dwu, h, workspace,
                            workspace_bytes=None, stream=None):
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load().samd_gated_ffn_backward(ctypes.byref(desc), _ptr(dh), _block8(ckpt_x), _block8(ckpt_g),
                                          _block8(ckpt_u), _ptr(wg), _ptr(wu), _ptr(dx), _ptr(dwg), _ptr(dwu), _ptr(h),
                                          _ptr(workspace), nb, _stream(stream)), "samd_gated_ffn_backward")


def samd_cache_append(cache: samd_cache, seqs: samd_cache_seqs, starts, tokens, k, ldk, v, ldv, stream=None):
    _check(load().samd_cache_append(ctypes.byref(cache), ctypes.byref(seqs), _ptr(starts), tokens, _ptr(k), ldk, _ptr(v),
                                    ldv, _stream(stream)), "samd_cache_append")


def samd_cache_read(cache: samd_cache, seqs: samd_cache_seqs, starts, tokens, k, ldk, v, ldv, stream=None):
    _check(load().samd_cache_read(ctypes.byref(cache), ctypes.byref(seqs), _ptr(starts), tokens, _ptr(k), ldk, _ptr(v),
                                  ldv, _stream(stream)), "samd_cache_read")


def samd_paged_attention_workspace_size(cache: samd_cache, seqs: samd_cache_seqs, q_heads: int, scores: bool) -> int:
    return int(load().samd_paged_attention_workspace_size(ctypes.byref(cache), ctypes.byref(seqs), q_heads, int(scores)))


def samd_paged_attention(cache: samd_cache, seqs: samd_cache_seqs, q_heads, q, ldq, scale, out, ldo, scores, ld_scores,
                         workspace, workspace_bytes=None, stream=None):
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load().samd_paged_attention(ctypes.byref(cache), ctypes.byref(seqs), q_heads, _ptr(q), ldq, scale, _ptr(out),
                                       ldo, _ptr(scores), ld_scores, _ptr(workspace), nb, _stream(stream)),
           "samd_paged_attention")


def samd_cache_evict(cache: samd_cache, seqs: samd_cache_seqs, scores, ld_scores, keep, recent, dst_table, ld_dst, kept,
                     new_lengths, new_scores, stream=None):
    _check(load().samd_cache_evict(ctypes.byref(cache), ctypes.byref(seqs), _ptr(scores), ld_scores, keep, recent,
                                   _ptr(dst_table), ld_dst, _ptr(kept), _ptr(new_lengths), _ptr(new_scores),
                                   _stream(stream)), "samd_cache_evict")


def samd_moe_route(desc: samd_moe_desc, normalize, x, router, ids, weights, stream=None):
    _check(load().samd_moe_route(ctypes.byref(desc), int(normalize), _ptr(x), _ptr(router), _ptr(ids), _ptr(weights),
                                 _stream(stream)), "samd_moe_route")


def samd_moe4_workspace_size(desc: samd_moe_desc) -> int:
    return int(load().samd_moe4_workspace_size(ctypes.byref(desc)))


def samd_moe4(desc: samd_moe_desc, fw, x, ids, weights, gate, up, down, y, workspace, workspace_bytes=None, stream=None):
    """gate, up, down: (lanes, scales, zeros or None)."""
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load().samd_moe4(ctypes.byref(desc), fw, _ptr(x), _ptr(ids), _ptr(weights), _weights4(*gate), _weights4(*up),
                            _weights4(*down), _ptr(y), _ptr(workspace), nb, _stream(stream)), "samd_moe4")


def samd_device_status(reset: bool = False, stream=None) -> int:
    v = ctypes.c_int(0)
    _check(load().samd_device_status(ctypes.byref(v), int(reset), _stream(stream)), "samd_device_status")
    return v.value


def samd_selftest_wait_timeout(limit_ns: int, stream=None) -> None:
    _check(load().samd_selftest_wait_timeout(limit_ns, _stream(stream)), "samd_selftest_wait_timeout")


def samd_version() -> str:
    return load().samd_version().decode()


# ---- allocating helpers ---------------------------------------------------------


def empty_words(f: samd_fmt, rows: int, inner: int, device="cuda") -> torch.Tensor:
    n = samd_packed_words(f, rows, inner)
    if n < 0:
        raise ValueError(f"bad format {f}")
    return torch.empty(max(n, 1), dtype=word_dtype(f), device=device)[:n]


def pack(x: torch.Tensor, f: samd_fmt, rows: int | None = None, inner: int | None = None, stream=None):
    """int8 tensor (rows x inner, row-major) -> packed words."""
    x = x.contiguous()
    if rows is None:
        inner = x.shape[-1] if x.dim() else 1
        rows = x.numel() // max(inner, 1)
    out = empty_words(f, rows, inner, x.device)
    samd_pack(f, x, out, rows, inner, stream)
    return out


def unpack(words: torch.Tensor, f: samd_fmt, rows: int, inner: int, stream=None) -> torch.Tensor:
    out = torch.empty(rows * inner, dtype=torch.int8, device=words.device)
    samd_unpack(f, words, out, rows, inner, stream)
    return out.view(rows, inner)


def elementwise(op, a, b, fa: samd_fmt, n: int, fo: samd_fmt | None = None, shift: int = 0, saturate: bool = False,
                out=None, stream=None):
    fo = fa if fo is None else fo
    if out is None:
        out = empty_words(fo, 1, n, a.device)
    samd_elementwise(op, fa, a, b, fo, out, n, shift, saturate, stream)
    return out


@dataclass
class ConvShape:
    N: int
    C: int
    H: int
    W: int
    K: int
    R: int = 3
    S: int = 3
    stride: int = 1
    pad: int = 1

    @property
    def Ho(self):
        return (self.H + 2 * self.pad - self.R) // self.stride + 1

    @property
    def Wo(self):
        return (self.W + 2 * self.pad - self.S) // self.stride + 1

    @property
    def macs(self) -> int:
        return self.N * self.Ho * self.Wo * self.K * self.C * self.R * self.S

    def desc(self, layout=SAMD_NHWC) -> samd_conv_desc:
        return samd_conv_desc(self.N, self.C, self.H, self.W, self.K, self.R, self.S, self.stride, self.pad, layout)


def conv_workspace(shape: ConvShape, fa: samd_fmt, fw: samd_fmt, device="cuda") -> torch.Tensor:
    nbytes = samd_conv2d_workspace_size(shape.desc(), fa, fw)
    if nbytes == 0:
        raise ValueError("invalid convolution shape or format")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def conv2d(act, wt, shape: ConvShape, fa: samd_fmt, fw: samd_fmt, fo: samd_fmt | None = None, shift: int = 0,
           want_acc: bool = True, workspace=None, stream=None):
    """NHWC packed conv; returns (int32 acc [N,Ho,Wo,K] or None, packed output words or None)."""
    dev = act.device
    acc = torch.empty((shape.N, shape.Ho, shape.Wo, shape.K), dtype=torch.int32, device=dev) if want_acc else None
    packed = empty_words(fo, shape.N * shape.Ho * shape.Wo, shape.K, dev) if fo is not None else None
    if workspace is None:
        workspace = conv_workspace(shape, fa, fw, dev)
    samd_conv2d(shape.desc(), fa, act, fw, wt, acc, fo, packed, shift, workspace, stream=stream)
    return acc, packed


def conv2d_nchw(act, wt, shape: ConvShape, fa: samd_fmt, fw: samd_fmt, fo: samd_fmt | None = None, shift: int = 0,
                want_acc: bool = True, workspace=None, stream=None):
    """NCHW packed along W (rows of W lanes; weights [K][C][R] rows of S lanes);
    returns (int32 acc [N,K,Ho,Wo] or None, packed output rows of Wo lanes or None)."""
    dev = act.device
    desc = shape.desc(SAMD_NCHW)
    acc = torch.empty((shape.N, shape.K, shape.Ho, shape.Wo), dtype=torch.int32, device=dev) if want_acc else None
    packed = empty_words(fo, shape.N * shape.K * shape.Ho, shape.Wo, dev) if fo is not None else None
    if workspace is None:
        nbytes = samd_conv2d_workspace_size(desc, fa, fw)
        if nbytes == 0:
            raise SamdError(SAMD_EUNSUP, "samd_conv2d_workspace_size")
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    samd_conv2d(desc, fa, act, fw, wt, acc, fo, packed, shift, workspace, stream=stream)
    return acc, packed


class PreparedConv:
    """A convolution layer whose weights were widened once (samd_conv2d_prepare)."""

    def __init__(self, wt_words, shape: ConvShape, fa: samd_fmt, fw: samd_fmt, fo: samd_fmt | None = None,
                 stream=None):
        self.shape, self.fa, self.fw, self.fo = shape, fa, fw, fo
        self.prepared = conv_workspace(shape, fa, fw, wt_words.device)
        samd_conv2d_prepare(shape.desc(), fa, fw, wt_words, fo, self.prepared, stream=stream)

    def __call__(self, act, acc_out=None, packed_out=None, shift: int = 0, stream=None):
        samd_conv2d_prepared(self.shape.desc(), self.fa, act, self.fw, self.prepared, acc_out, self.fo, packed_out,
                             shift, stream=stream)
        return acc_out, packed_out

    def pool2x2_supported(self) -> bool:
        return self.fo is not None and samd_conv2d_pool2x2_supported(self.shape.desc(), self.fa, self.fw, self.fo)

    def pool2x2(self, act, pooled_out, shift: int = 0, stream=None):
        """The convolution with the 2x2 max-pool of its packed output fused
        (samd_conv2d_prepared_pool2x2)."""
        samd_conv2d_prepared_pool2x2(self.shape.desc(), self.fa, act, self.fw, self.prepared, self.fo, pooled_out,
                                     shift, stream=stream)
        return pooled_out

    def outputs(self, want_acc=True, want_packed=True, device="cuda"):
        s = self.shape
        acc = torch.empty((s.N, s.Ho, s.Wo, s.K), dtype=torch.int32, device=device) if want_acc else None
        packed = empty_words(self.fo, s.N * s.Ho * s.Wo, s.K, device) if (want_packed and self.fo) else None
        return acc, packed


def maxpool2x2(words, f: samd_fmt, N: int, C: int, H: int, W: int, stream=None):
    out = empty_words(f, N * (H // 2) * (W // 2), C, words.device)
    samd_maxpool2x2(f, words, out, N, C, H, W, SAMD_NHWC, stream)
    return out


# ---- the gated feed-forward block -------------------------------------------------


_HERE = contextlib.nullcontext()


def _on(stream):
    """Allocations made inside belong to the stream that uses them."""
    if stream is None:
        return _HERE
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


def _rows(t: torch.Tensor, what: str, cols: int | None = None, rows: int | None = None, dtype=None) -> int:
    """Checks a matrix whose rows lie contiguous in memory and returns its row stride in elements."""
    shape = t.shape
    if cols is None and len(shape) == 2 and t.is_contiguous():
        return max(shape[1], 1)
    if len(shape) != 2 or (shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: a matrix with contiguous rows is wanted, got shape {tuple(shape)}, "
                         f"strides {t.stride()}")
    if (cols is not None and shape[1] != cols) or (rows is not None and shape[0] != rows):
        raise ValueError(f"{what}: shape {tuple(shape)}, wanted ({rows if rows is not None else 'any'}, "
                         f"{cols if cols is not None else 'any'})")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what}: {t.dtype}, wanted {dtype}")
    return t.stride(0) if shape[0] > 1 else max(shape[1], 1)


def _check_weights4(lanes, scales, zeros, N, K, group, f, dtype):
    shape = (N, -(-K // group))
    if lanes.dtype != word_dtype(f) or not lanes.is_contiguous() or lanes.numel() != N * -(-K // (f.word_bits // 4)):
        raise ValueError(f"lanes: {N} packed rows of {K} 4-bit lanes are wanted")
    if scales.dtype != dtype or scales.shape != shape or not scales.is_contiguous():
        raise ValueError(f"scales: a contiguous {shape} {dtype} tensor is wanted")
    if zeros is not None and (zeros.dtype != torch.uint8 or zeros.shape != shape or not zeros.is_contiguous()):
        raise ValueError(f"zeros: a contiguous {shape} uint8 tensor is wanted")


def _past_int(*sizes: int):
    """The descriptors' sizes are C ints, and ctypes cuts what does not fit one."""
    raise ValueError(f"a size of {max(sizes)}: the library's matrix products take sizes below 2^31 at most")


def _matvec_desc(x, scales, group, out):
    t = x.dtype
    if t is not torch.float16 and t is not torch.bfloat16:
        raise ValueError(f"x: {t}, wanted float16 or bfloat16")
    if group < 32 or group & (group - 1):
        raise ValueError(f"group: {group}, wanted a power of two of at least 32")
    ldx = _rows(x, "x")
    (M, K), N = x.shape, scales.shape[0]
    if (M | K | N) >> 31:
        _past_int(M, K, N)
    return samd_matvec_desc(M, N, K, group, ldx, N if out is None else _rows(out, "out", N, M, t), DTYPES[t])


def matvec4(x, lanes, scales, group: int, f: samd_fmt, zeros=None, out=None, stream=None):
    """x (M, K) times N rows of K packed 4-bit weights, scales (N, ceil(K / group)) of x's type and, for unsigned
    lanes, zero points of the same shape (uint8): out (M, N), y = x @ (scale * (lane - zero)).T."""
    d = _matvec_desc(x, scales, group, out)
    _check_weights4(lanes, scales, zeros, d.N, d.K, group, f, x.dtype)
    if out is None:
        out = _empty(x, d.M, d.N, stream)
    samd_matvec4(d, f, x, lanes, scales, zeros, out, stream)
    return out


def gated_matvec4(x, lanes_g, scales_g, lanes_u, scales_u, group: int, f: samd_fmt, act="silu", zeros_g=None,
                  zeros_u=None, out=None, stream=None):
    """act(x @ Wg.T) * (x @ Wu.T) over two sets of packed 4-bit weights, as matvec4 takes one."""
    d = _matvec_desc(x, scales_g, group, out)
    _check_weights4(lanes_g, scales_g, zeros_g, d.N, d.K, group, f, x.dtype)
    _check_weights4(lanes_u, scales_u, zeros_u, d.N, d.K, group, f, x.dtype)
    if out is None:
        out = _empty(x, d.M, d.N, stream)
    samd_gated_matvec4(d, act, f, x, (lanes_g, scales_g, zeros_g), (lanes_u, scales_u, zeros_u), out, stream)
    return out


def _empty(like, rows: int, cols: int, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty((rows, cols), dtype=like.dtype, device=like.device)
    with _on(stream):
        return torch.empty((rows, cols), dtype=like.dtype, device=like.device)


class Block8:
    """An activation tensor of `rows` rows of `inner` elements in 8 bits (samd_block8): lanes, the packed rows (int32,
    format block8_fmt()), and exps, the block exponents (uint8). block8_empty puts both into one allocation, of which
    the two tensors are views that are made when they are asked for."""

    __slots__ = ("rows", "inner", "_lanes", "_exps", "_buf")

    def __init__(self, lanes: torch.Tensor | None, exps: torch.Tensor | None, inner: int, rows: int | None = None,
                 buf: torch.Tensor | None = None):
        self.rows, self.inner = lanes.shape[0] if rows is None else rows, inner
        self._lanes, self._exps, self._buf = lanes, exps, buf

    def _lane_words(self) -> int:
        """Words of all rows, up to the exponents of a block8_empty (16-byte units)."""
        return -(-self.rows * -(-self.inner // 4) // 4) * 4

    @property
    def lanes(self) -> torch.Tensor:
        if self._lanes is None:
            words = -(-self.inner // 4)
            self._lanes = self._buf[:self.rows * words].view(self.rows, words)
        return self._lanes

    @property
    def exps(self) -> torch.Tensor:
        if self._exps is None:
            n = -(-self.inner // 32)
            self._exps = self._buf[self._lane_words():].view(torch.uint8)[:self.rows * n].view(self.rows, n)
        return self._exps

    def __getitem__(self, i):
        return (self.lanes, self.exps)[i]


def block8_fmt() -> samd_fmt:
    return fmt(8, True, 0, 32)


def block8_empty(rows: int, inner: int, device="cuda") -> Block8:
    b = Block8(None, None, inner, rows)
    b._buf = torch.empty(b._lane_words() + -(-rows * -(-inner // 32) // 4), dtype=torch.int32, device=device)
    return b


def _check_block8(b: Block8, what: str, rows: int, inner: int):
    if b.rows != rows or b.inner != inner:
        raise ValueError(f"{what}: the 8-bit form of a ({rows}, {inner}) tensor is wanted, got ({b.rows}, {b.inner})")
    if b._buf is None and (b.lanes.shape != (rows, -(-inner // 4)) or b.exps.shape != (rows, -(-inner // 32)) or
                           not b.lanes.is_contiguous() or not b.exps.is_contiguous() or
                           b.lanes.dtype != torch.int32 or b.exps.dtype != torch.uint8):
        raise ValueError(f"{what}: contiguous int32 lanes and uint8 exponents of a ({rows}, {inner}) tensor are wanted")


def block8_quantize(x: torch.Tensor, out: Block8 | None = None, stream=None) -> Block8:
    """The 8-bit form of a matrix (float16, bfloat16 or float32)."""
    if x.dtype not in DTYPES:
        raise ValueError(f"x: {x.dtype}, wanted float16, bfloat16 or float32")
    ldx = _rows(x, "x")
    rows, inner = x.shape
    if out is None:
        with _on(stream):
            out = block8_empty(rows, inner, x.device)
    else:
        _check_block8(out, "out", rows, inner)
    samd_block8_quantize(x.dtype, x, ldx, rows, inner, out, stream)
    return out


def block8_dequantize(b: Block8, dtype: torch.dtype, out=None, stream=None) -> torch.Tensor:
    """The values an 8-bit form stands for, as a matrix of `dtype`."""
    if dtype not in DTYPES:
        raise ValueError(f"dtype: {dtype}, wanted float16, bfloat16 or float32")
    rows, inner = b.rows, b.inner
    _check_block8(b, "b", rows, inner)
    if out is None:
        with _on(stream):
            out = torch.empty((rows, inner), dtype=dtype, device=(b._lanes if b._buf is None else b._buf).device)
        ldy = max(inner, 1)
    else:
        ldy = _rows(out, "out", inner, rows, dtype)
    samd_block8_dequantize(dtype, b, rows, inner, out, ldy, stream)
    return out


def _aligned8(n: int) -> int:
    return -(-n // 8) * 8


def _empty_ld(rows: int, cols: int, ld: int, like: torch.Tensor) -> torch.Tensor:
    """A (rows, cols) matrix of `like`'s type whose rows start ld elements apart."""
    if ld == cols:
        return torch.empty((rows, cols), dtype=like.dtype, device=like.device)
    return torch.empty_strided((rows, cols), (ld, 1), dtype=like.dtype, device=like.device)


def _ffn_desc(M, K, F, t, act, ldx, ldw, ldh) -> samd_ffn_desc:
    if t not in (torch.float16, torch.bfloat16):
        raise ValueError(f"{t}: float16 or bfloat16 is wanted")
    if (M | K | F) >> 31:
        _past_int(M, K, F)
    return samd_ffn_desc(M, K, F, ldx, ldw, ldh, DTYPES[t], _act(act))


def _ld8(t: torch.Tensor, what: str, rows: int, cols: int, dtype) -> int:
    """The row stride of a matrix of the block, rounded up where a single row leaves it open."""
    if cols % 8 == 0 and t.dtype is dtype and t.shape == (rows, cols) and t.is_contiguous():
        return cols
    ld = _rows(t, what, cols, rows, dtype)
    return ld if rows > 1 else _aligned8(ld)


def _same_ld(a: int, b: int, what: str) -> int:
    if a != b:
        raise ValueError(f"{what}: one row stride for both is wanted, got {a} and {b}")
    return a


def gated_ffn_forward(x, wg, wu, act="silu", checkpoints: bool = False, out=None, stream=None):
    """h = act(x @ wg.T) * (x @ wu.T) for x (M, K), wg and wu (F, K), whose rows start 16-byte units apart (a row
    stride that is a multiple of 8). With checkpoints: (h, ckpt_g, ckpt_u), the two products in 8 bits for
    gated_ffn_backward."""
    (M, K), F, t = x.shape, wg.shape[0], x.dtype
    ldx, ldw = _ld8(x, "x", M, K, t), _same_ld(_ld8(wg, "wg", F, K, t), _ld8(wu, "wu", F, K, t), "wg, wu")
    ldh = _aligned8(F) if out is None else _ld8(out, "out", M, F, t)
    d = _ffn_desc(M, K, F, t, act, ldx, ldw, ldh)
    with _on(stream):
        h = _empty_ld(M, F, ldh, x) if out is None else out
        if not checkpoints:
            samd_gated_ffn_forward(d, x, wg, wu, h, None, None, stream)
            return h
        g8, u8 = block8_empty(M, F, x.device), block8_empty(M, F, x.device)
        samd_gated_ffn_forward(d, x, wg, wu, h, g8, u8, stream)
        return h, g8, u8


def gated_ffn_backward(dh, ckpt_x: Block8, ckpt_g: Block8, ckpt_u: Block8, wg, wu, act="silu", need_dx: bool = True,
                       need_dw: bool = True, need_h: bool = False, workspace=None, stream=None):
    """Gradients of gated_ffn_forward from dh (M, F) and the 8-bit forms of x, g and u: (dx, dwg, dwu), None for those
    not wanted, and with need_h also h formed again from the checkpoints (for the next layer's weight gradient)."""
    (M, F), K, t = dh.shape, wg.shape[1], dh.dtype
    if need_dw:
        _check_block8(ckpt_x, "ckpt_x", M, K)
    _check_block8(ckpt_g, "ckpt_g", M, F)
    _check_block8(ckpt_u, "ckpt_u", M, F)
    ldw = _same_ld(_ld8(wg, "wg", F, K, t), _ld8(wu, "wu", F, K, t), "wg, wu")
    ldh = _ld8(dh, "dh", M, F, t)
    d = _ffn_desc(M, K, F, t, act, _aligned8(K), ldw, ldh)
    if not (need_dx or need_dw or need_h):
        raise ValueError("nothing is wanted")
    with _on(stream):
        dx = _empty_ld(M, K, d.ldx, dh) if need_dx else None
        dwg, dwu = (_empty_ld(F, K, ldw, dh), _empty_ld(F, K, ldw, dh)) if need_dw else (None, None)
        h = _empty_ld(M, F, ldh, dh) if need_h else None
        if workspace is None:
            workspace = torch.empty(samd_gated_ffn_backward_workspace_size(d), dtype=torch.uint8, device=dh.device)
        samd_gated_ffn_backward(d, dh, ckpt_x, ckpt_g, ckpt_u, wg, wu, dx, dwg, dwu, h, workspace, stream=stream)
    return (dx, dwg, dwu, h) if need_h else (dx, dwg, dwu)


# ---- the packed key-value cache ----------------------------------------------------
#
# A decoder makes these calls for every layer and token, and the smallest ones take less time on the GPU than their checks
# here: a call first asks whether all is as it has to be, and only then what is not.


def _address(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("libsamd takes device tensors")
    return t.data_ptr()


# samd_cache and samd_cache_seqs, laid out as C lays them out: half the time of a structure's constructor
_CACHE_BYTES = struct.Struct("@4i4BiQQQQ").pack
_SEQS_BYTES = struct.Struct("@iiqQQ").pack


class PagedCache:
    """Keys and values of tokens in packed lanes, in pages (samd_cache): k_lanes and v_lanes (pages, heads, page, words)
    int32, the rows as samd_pack writes them in the format cache_fmt(bits); k_scales and v_scales (pages, heads, page,
    dim // 32) float16 or bfloat16. The lane width follows from the shapes."""

    __slots__ = ("k_lanes", "k_scales", "v_lanes", "v_scales", "bits", "dim", "heads", "page", "dtype", "_desc")

    def __init__(self, k_lanes, k_scales, v_lanes, v_scales):
        lanes, scales, t = k_lanes.shape, k_scales.shape, k_scales.dtype
        if (len(lanes) != 4 or lanes[:3] != scales[:-1] or v_lanes.shape != lanes or v_scales.shape != scales or
                (t is not torch.bfloat16 and t is not torch.float16) or v_scales.dtype is not t or
                k_lanes.dtype is not torch.int32 or v_lanes.dtype is not torch.int32 or not k_lanes.is_contiguous() or
                not k_scales.is_contiguous() or not v_lanes.is_contiguous() or not v_scales.is_contiguous()):
            raise ValueError(f"contiguous int32 lanes (pages, heads, page, words) and float16 or bfloat16 scales (pages, heads, "
                             f"page, dim // 32) are wanted, the same for keys and values, got {tuple(lanes)}, {tuple(scales)}, "
                             f"{tuple(v_lanes.shape)}, {tuple(v_scales.shape)} of {t}")
        pages, heads, page, words = lanes
        blocks = scales[3]
        bits = words // blocks if blocks else 0
        if bits not in (4, 8) or bits * blocks != words:
            raise ValueError(f"rows of {words} words with {blocks} scales: 4 or 8 of them for a scale are wanted")
        if (pages | heads | page) >> 31:
            _past_int(pages, heads, page)
        self.k_lanes, self.k_scales, self.v_lanes, self.v_scales = k_lanes, k_scales, v_lanes, v_scales
        self.bits, self.dim, self.heads, self.page, self.dtype = bits, 32 * blocks, heads, page, t
        self._desc = samd_cache.from_buffer_copy(_CACHE_BYTES(
            pages, page, heads, 32 * blocks, bits, 1, 0, 32, DTYPES[t], _address(k_lanes), _address(k_scales),
            _address(v_lanes), _address(v_scales)))


def cache_fmt(bits: int) -> samd_fmt:
    return fmt(bits, True, 0, 32)


def cache_empty(pages: int, page: int, heads: int, dim: int, bits: int, dtype: torch.dtype, device="cuda") -> PagedCache:
    """A cache of `pages` pages of `page` tokens (a power of two, 16 or more) for `heads` key heads of `dim` elements (a
    multiple of 32 up to 256), in lanes of `bits` (4 or 8). Its rows are not initialised: none is read that was not
    written, as long as the sequences' lengths count what was."""
    if bits not in (4, 8) or dim % 32 or not 32 <= dim <= 256 or page < 16 or page & (page - 1):
        raise ValueError(f"page {page}, dim {dim}, bits {bits}: a power of two of at least 16, a multiple of 32 up to 256, "
                         "and 4 or 8 are wanted")
    def lanes():
        return torch.empty((pages, heads, page, dim * bits // 32), dtype=torch.int32, device=device)
    def scales():
        return torch.empty((pages, heads, page, dim // 32), dtype=dtype, device=device)
    return PagedCache(lanes(), scales(), lanes(), scales())


def _cache_seqs(table, lengths) -> samd_cache_seqs:
    """table (sequences, pages of one) int32 with contiguous rows, lengths (sequences) int32."""
    if table.dtype is not torch.int32 or lengths.dtype is not torch.int32:
        raise ValueError(f"table, lengths: {table.dtype}, {lengths.dtype}, wanted int32")
    ld = _rows(table, "table")
    seqs, width = table.shape
    if lengths.shape != (seqs,) or not lengths.is_contiguous():
        raise ValueError(f"lengths: a contiguous ({seqs},) tensor is wanted, got {tuple(lengths.shape)}")
    if (seqs | width) >> 31:
        _past_int(seqs, width)
    return samd_cache_seqs.from_buffer_copy(_SEQS_BYTES(seqs, width, ld, _address(table), _address(lengths)))


def _token_rows(x, what: str, heads: int, dim: int, dtype, tokens: int | None = None) -> int:
    """Checks a (tokens, heads, dim) tensor whose tokens lie whole in memory, and returns the stride of a token."""
    shape = x.shape
    if (x.dtype is dtype and len(shape) == 3 and shape[1] == heads and shape[2] == dim and
            (tokens is None or shape[0] == tokens) and x.is_contiguous()):
        return heads * dim
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or (tokens is not None and shape[0] != tokens):
        raise ValueError(f"{what}: shape {tuple(shape)}, wanted ({tokens if tokens is not None else 'any'}, {heads}, {dim})")
    if x.dtype is not dtype:
        raise ValueError(f"{what}: {x.dtype}, wanted {dtype}")
    if x.stride(2) != 1 or (heads > 1 and x.stride(1) != dim):
        raise ValueError(f"{what}: the heads of a token one behind the other are wanted, got strides {x.stride()}")
    return x.stride(0) if shape[0] > 1 else heads * dim


def _starts(starts, seqs: int):
    if starts is not None and (starts.dtype is not torch.int32 or starts.shape != (seqs + 1,) or not starts.is_contiguous()):
        raise ValueError(f"starts: a contiguous ({seqs + 1},) int32 tensor is wanted")
    return starts


def _scores_ld(scores, seqs: int, heads: int) -> int:
    if (scores.dtype is not torch.float32 or scores.dim() != 3 or scores.shape[0] != seqs or scores.shape[1] != heads or
            not scores.is_contiguous()):
        raise ValueError(f"scores: a contiguous ({seqs}, {heads}, any) float32 tensor is wanted")
    return scores.shape[2]


def _new(like, shape, dtype, stream) -> torch.Tensor:
    """An uninitialised tensor on the device of `like`, of the stream that is going to use it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with _on(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def cache_append(cache: PagedCache, k, v, table, lengths, starts=None, stream=None) -> None:
    """Writes new tokens' keys and values (tokens, heads, dim) into the cache. lengths counts them already: rows
    starts[b] .. starts[b + 1] - 1 are the last tokens of sequence b; without starts every sequence has one, row b."""
    heads, dim, t = cache.heads, cache.dim, cache.dtype
    ldk = _token_rows(k, "k", heads, dim, t)
    tokens = k.shape[0]
    ldv = _token_rows(v, "v", heads, dim, t, tokens)
    s = _cache_seqs(table, lengths)
    if tokens >> 31:
        _past_int(tokens)
    samd_cache_append(cache._desc, s, _starts(starts, s.seqs), tokens, k, ldk, v, ldv, stream)


def cache_read(cache: PagedCache, tokens: int, table, lengths, starts=None, k=None, v=None, stream=None):
    """(k, v): the values (tokens, heads, dim) of the rows that cache_append with the same table, lengths and starts
    wrote, in the scales' type. Rows of no sequence are left as they are in k and v."""
    heads, dim, t = cache.heads, cache.dim, cache.dtype
    s = _cache_seqs(table, lengths)
    if not 0 <= tokens < 1 << 31:
        _past_int(tokens)
    ldk = ldv = heads * dim
    if k is None:
        k = _new(cache.k_scales, (tokens, heads, dim), t, stream)
    else:
        ldk = _token_rows(k, "k", heads, dim, t, tokens)
    if v is None:
        v = _new(cache.k_scales, (tokens, heads, dim), t, stream)
    else:
        ldv = _token_rows(v, "v", heads, dim, t, tokens)
    samd_cache_read(cache._desc, s, _starts(starts, s.seqs), tokens, k, ldk, v, ldv, stream)
    return k, v


@functools.lru_cache(maxsize=1024)
def _attention_workspace(device: int, pages, page, heads, dim, bits, seqs, max_pages, q_heads, scores) -> int:
    """Bytes of workspace by the current device, whose SMs the library goes by, and sizes alone: they are the same for
    every layer of a model."""
    c = samd_cache(pages, page, heads, dim, cache_fmt(bits), SAMD_F16, None, None, None, None)
    return samd_paged_attention_workspace_size(c, samd_cache_seqs(seqs, max_pages, max_pages, None, None), q_heads, scores)


def paged_attention(q, cache: PagedCache, table, lengths, scale: float | None = None, scores=None, out=None,
                    workspace=None, stream=None):
    """One query token for each sequence over the cache: q and out (sequences, query heads, dim), key head h for a run of
    query heads; scale defaults to dim ** -0.5. scores (sequences, heads, any) float32: each token's weight is added to
    it, for cache_evict."""
    s = _cache_seqs(table, lengths)
    seqs, heads, dim = s.seqs, cache.heads, cache.dim
    q_heads = q.shape[1] if q.dim() == 3 else 0
    ldq = _token_rows(q, "q", q_heads, dim, cache.dtype, seqs)
    if q_heads < 1 or q_heads % heads or q_heads >> 31:
        raise ValueError(f"q: {q_heads} heads, wanted a multiple of the cache's {heads}")
    ld_scores = 0 if scores is None else _scores_ld(scores, seqs, heads)
    if out is None:
        out, ldo = _new(q, (seqs, q_heads, dim), cache.dtype, stream), q_heads * dim
    else:
        ldo = _token_rows(out, "out", q_heads, dim, q.dtype, seqs)
    nb = None
    if workspace is None:
        nb = _attention_workspace(torch.cuda.current_device(), cache._desc.pages, cache.page, heads, dim, cache.bits, seqs,
                                  s.max_pages, q_heads, ld_scores > 0)
        workspace = _new(q, (nb,), torch.uint8, stream) if nb else None
    samd_paged_attention(cache._desc, s, q_heads, q, ldq, dim ** -0.5 if scale is None else scale, out, ldo,
                         scores if ld_scores else None, ld_scores, workspace, nb, stream)
    return out


def cache_evict(cache: PagedCache, table, lengths, scores, dst_table, keep: int, recent: int = 0, stream=None):
    """Cuts every head of every sequence down to `keep` tokens, its last `recent` ones and those with the largest scores
    (sequences, heads, any), by copying the kept rows, in order, into the pages of dst_table (other ones than the
    sequences'). (kept, new lengths, new scores): the kept tokens' places (sequences, heads, keep), -1 behind the last,
    and their scores, 0 behind it; dst_table with the new lengths and scores is the cache to go on with."""
    s = _cache_seqs(table, lengths)
    seqs, heads = s.seqs, cache.heads
    ld_scores = _scores_ld(scores, seqs, heads)
    if not 0 <= recent <= keep or keep < 1:
        raise ValueError(f"keep {keep}, recent {recent}: 0 <= recent <= keep, and a keep of 1 or more, are wanted")
    if keep >> 31:
        _past_int(keep)
    if dst_table.dtype is not torch.int32 or dst_table.shape[0] != seqs or dst_table.shape[1] * cache.page < keep:
        raise ValueError(f"dst_table: ({seqs}, {-(-keep // cache.page)}) int32 pages are wanted")
    ld_dst = _rows(dst_table, "dst_table")
    kept = _new(scores, (seqs, heads, keep), torch.int32, stream)
    new_lengths = _new(scores, (seqs,), torch.int32, stream)
    new_scores = _new(scores, (seqs, heads, keep), torch.float32, stream)
    samd_cache_evict(cache._desc, s, scores, ld_scores, keep, recent, dst_table, ld_dst, kept, new_lengths, new_scores, stream)
    return kept, new_lengths, new_scores


# ---- a layer of experts ----------------------------------------------------------------


def _moe_desc(x, E: int, topk: int, F: int = 32, group: int = 32, ldy: int = 0, act="silu") -> samd_moe_desc:
    t = x.dtype
    if t is not torch.float16 and t is not torch.bfloat16:
        raise ValueError(f"x: {t}, wanted float16 or bfloat16")
    if not 1 <= topk <= 32:
        raise ValueError(f"{topk} experts of a token: 1 .. 32 are wanted")
    if group < 32 or group & (group - 1):
        raise ValueError(f"group: {group}, wanted a power of two of at least 32")
    M, K = x.shape
    ldx = _ld8(x, "x", M, K, t)
    if (M | K | E | F | group) >> 31:
        _past_int(M, K, E, F, group)
    return samd_moe_desc(M, K, F, E, topk, group, ldx, ldy or K, DTYPES[t], _act(act))


def _check_router(router, x, topk: int) -> None:
    if router.dtype is not x.dtype or router.dim() != 2 or router.shape[1] != x.shape[-1] or not router.is_contiguous():
        raise ValueError(f"router: a contiguous (experts, {x.shape[-1]}) {x.dtype} tensor is wanted")
    if topk > router.shape[0]:
        raise ValueError(f"{topk} experts of {router.shape[0]} are wanted")


def moe_route(x, router, topk: int, normalize: bool = True, ids=None, weights=None, stream=None):
    """(ids, weights), (M, topk) int32 and float32: the experts with the largest logits of x (M, K) by router (E, K), the
    largest first, and the softmax of their logits, over themselves (normalize) or over all experts."""
    _check_router(router, x, topk)
    d = _moe_desc(x, router.shape[0], topk)
    for o, what, t in ((ids, "ids", torch.int32), (weights, "weights", torch.float32)):
        if o is not None and (o.dtype is not t or o.shape != (d.M, topk) or not o.is_contiguous()):
            raise ValueError(f"{what}: a contiguous ({d.M}, {topk}) {t} tensor is wanted")
    if ids is None:
        ids = _new(x, (d.M, topk), torch.int32, stream)
    if weights is None:
        weights = _new(x, (d.M, topk), torch.float32, stream)
    samd_moe_route(d, normalize, x, router, ids, weights, stream)
    return ids, weights


def _are_weights4(w, rows: int, groups: int, words: int, word, dtype) -> bool:
    lanes, scales = w[0], w[1]
    if (lanes.dtype is not word or scales.dtype is not dtype or scales.shape != (rows, groups) or lanes.numel() != rows * words or
            not lanes.is_contiguous() or not scales.is_contiguous()):
        return False
    zeros = w[2] if len(w) > 2 else None
    return zeros is None or (zeros.dtype is torch.uint8 and zeros.shape == (rows, groups) and zeros.is_contiguous())


def _experts4(gate, up, down, K: int, group: int, f: samd_fmt, dtype) -> tuple[int, int]:
    """Checks the matrices of a layer of experts, and returns how many experts there are and their hidden columns. The
    scales (rows of all experts, groups of a row) say how many rows there are."""
    rows, n = gate[1].shape[0], down[1].shape[0]
    E = n // K if K else 0
    if E < 1 or n != E * K or rows % E or group < 1:
        raise ValueError(f"gate, down: scales of {rows} and {n} rows, wanted a multiple of the experts, and {K} times them")
    F, L, word = rows // E, f.word_bits // 4, word_dtype(f)
    gk, wk = -(-K // group), -(-K // L)
    if not (_are_weights4(gate, rows, gk, wk, word, dtype) and _are_weights4(up, rows, gk, wk, word, dtype) and
            _are_weights4(down, n, -(-F // group), -(-F // L), word, dtype)):
        for w, r, k in ((gate, rows, K), (up, rows, K), (down, n, F)):  # which, and what
            _check_weights4(w[0], w[1], w[2] if len(w) > 2 else None, r, k, group, f, dtype)
    return E, F


def moe4(x, ids, weights, gate, up, down, group: int, f: samd_fmt, act="silu", out=None, workspace=None, stream=None):
    """y (M, K) = sum over j of weights[:, j] * (act(x @ Wg.T) * (x @ Wu.T)) @ Wd.T with the matrices of expert ids[:, j]
    (an id that is no expert's counts nothing). gate, up and down are (lanes, scales) or (lanes, scales, zeros), as matvec4
    takes them: E * F, E * F and E * K packed rows, one expert behind the other."""
    M, K = x.shape
    E, F = _experts4(gate, up, down, K, group, f, x.dtype)
    topk = ids.shape[1] if ids.dim() == 2 else 0
    if ids.dtype is not torch.int32 or ids.shape != (M, topk) or not ids.is_contiguous():
        raise ValueError(f"ids: a contiguous ({M}, any) int32 tensor is wanted")
    if weights.dtype is not torch.float32 or weights.shape != ids.shape or not weights.is_contiguous():
        raise ValueError(f"weights: a contiguous {tuple(ids.shape)} float32 tensor is wanted")
    ldy = K if out is None else _ld8(out, "out", M, K, x.dtype)
    d = _moe_desc(x, E, topk, F, group, ldy, act)
    if out is None:
        out = _new(x, (M, K), x.dtype, stream)
    if workspace is None:
        workspace = _new(x, (samd_moe4_workspace_size(d),), torch.uint8, stream)
    samd_moe4(d, f, x, ids, weights, _three(gate), _three(up), _three(down), out, workspace, None, stream)
    return out


def _three(w):
    return w if len(w) > 2 else (*w, None)


def moe_layer4(x, router, topk: int, gate, up, down, group: int, f: samd_fmt, act="silu", normalize: bool = True, out=None,
               workspace=None, stream=None):
    """A whole layer of experts: moe_route, and moe4 on its choice."""
    M, K = x.shape
    E, F = _experts4(gate, up, down, K, group, f, x.dtype)
    _check_router(router, x, topk)
    if router.shape[0] != E:
        raise ValueError(f"router: {router.shape[0]} experts, wanted {E}")
    d = _moe_desc(x, E, topk, F, group, K if out is None else _ld8(out, "out", M, K, x.dtype), act)
    if out is None:
        out = _new(x, (M, K), x.dtype, stream)
    # the choice and, where the caller has none, the layer's workspace in one allocation
    part = -(-4 * M * topk // 128) * 128
    buf = _new(x, (2 * part + (samd_moe4_workspace_size(d) if workspace is None else 0),), torch.uint8, stream)
    at, nb = _address(buf), None
    if workspace is None:
        workspace, nb = at + 2 * part, buf.numel() - 2 * part
    samd_moe_route(d, normalize, x, router, at, at + part, stream)
    samd_moe4(d, f, x, at, at + part, _three(gate), _three(up), _three(down), out, workspace, nb, stream)
    return out
