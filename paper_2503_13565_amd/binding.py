"""Thin ctypes binding of ``include/mxfp4.h``: argument marshalling only, for the common call of a product through the
extension module ``_host``.

Every step of the path runs in the HIP kernels of ``libmxfp4_hip.so``; torch supplies device
memory and the current stream.  There is no fallback: if the library has not been built
(``python -m paper_2503_13565_amd.build``) the first call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import warnings
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmxfp4_hip.so")

PATH_AUTO, PATH_VALU_BITS, PATH_VALU_CVT, PATH_VALU_LUT, PATH_MFMA, PATH_VALU_REG, PATH_MFMA_GENERAL = 0, 1, 2, 3, 4, 5, 6

EXPORTS = [
    "mxfp4_direct_cast", "mxfp4_direct_cast_bits", "mxfp4_dequant", "mxfp4_dequant_hwcvt", "mxfp4_woq_gemm", "mxfp4_woq_gemm_path",
    "mxfp4_woq_gemm_workspace_bytes", "mxfp4_woq_gemm_ws", "mxfp4_woq_gemm_argmax_workspace_bytes", "mxfp4_woq_gemm_argmax", "mxfp4_woq_gemm_argmax_path",
    "mxfp4_bf16_gemm", "mxfp4_bf16_gemm_argmax_workspace_bytes", "mxfp4_bf16_gemm_argmax",
    "mxfp4_woq_gemm_verify", "mxfp4_bf16_gemm_verify",
    "mxfp4_woq_gemm_fused", "mxfp4_woq_gemm_grouped_workspace_bytes", "mxfp4_woq_gemm_grouped",
    "mxfp4_woq_gemm_argmax_noalloc_max_bytes", "mxfp4_woq_gemm_argmax_noalloc",
    "mxfp4_woq_gemm_chain_workspace_bytes", "mxfp4_woq_gemm_chain_init", "mxfp4_woq_gemm_chain",
    "mxfp4_e4m3_direct_cast", "mxfp4_e4m3_direct_cast_bits", "mxfp4_e4m3_dequant", "mxfp4_e4m3_woq_gemm",
    "mxfp4_e4m3_woq_gemm_argmax",
    "mxfp4_e2m3_direct_cast", "mxfp4_e2m3_direct_cast_bits", "mxfp4_e2m3_dequant", "mxfp4_e2m3_woq_gemm",
    "mxfp4_e2m3_woq_gemm_argmax",
    "mxfp4_fmt_block_bytes", "mxfp4_fmt_direct_cast", "mxfp4_fmt_direct_cast_bits", "mxfp4_fmt_dequant",
    "mxfp4_fmt_woq_gemm", "mxfp4_fmt_woq_gemm_argmax",
    "mxfp4_woq_gemm_t_workspace_bytes", "mxfp4_woq_gemm_t",
    "mxfp4_kv_append", "mxfp4_kv_read", "mxfp4_kv_attention_workspace_bytes", "mxfp4_kv_attention",
    "mxfp4_kv_fork", "mxfp4_kv_extend", "mxfp4_kv_release", "mxfp4_kv_compact", "mxfp4_kv_copy_pages",
    "mxfp4_tile_repack_q_bytes", "mxfp4_tile_repack_s_bytes", "mxfp4_tile_repack", "mxfp4_woq_gemm_tiled",
    "mxfp4_woq_gemm_tiled_ws",
    "mxfp4_woq_gemm_tiled_argmax", "mxfp4_woq_gemm_tiled_verify", "mxfp4_woq_gemm_tiled_fused",
    "mxfp4_diag_stream_read", "mxfp4_diag_stream_copy", "mxfp4_last_error", "mxfp4_version",
]

_lib = None

# What ``_host`` takes (csrc/host.cpp): plain tensors on the current device that pass every check below, outputs
# allocated by the call.  It answers None to everything else, and the checks here take the call.
_MX, _E4M3, _E2M3, _BF16, _TILED, _FMT = 0, 1, 2, 3, 4, 16


def _product(*args):
    load()                                          # (puts the extension's functions in the place of these three)
    return _product(*args)


def _verify(*args):
    load()
    return _verify(*args)


def _cast(w):
    load()
    return _cast(w)


class _Kv:
    """The extension's calls of the paged cache; None from them as from the three above."""
    append = read = attention = pages = compact = staticmethod(lambda *args: None)


_kv = None


def _kv_host():
    load()
    return _kv


class GemmDesc(ctypes.Structure):
    """``mxfp4_gemm_desc`` of the header, field for field."""
    _fields_ = [("x_bf16", ctypes.c_void_p), ("M", ctypes.c_int64), ("ldx", ctypes.c_int64),
                ("q_packed", ctypes.c_void_p), ("scales_e8m0", ctypes.c_void_p), ("N", ctypes.c_int64),
                ("K", ctypes.c_int64), ("bias_bf16", ctypes.c_void_p), ("residual_bf16", ctypes.c_void_p),
                ("ldr", ctypes.c_int64), ("y_bf16", ctypes.c_void_p), ("ldy", ctypes.c_int64),
                ("argmax_out", ctypes.c_void_p), ("max_out", ctypes.c_void_p),
                ("act", ctypes.c_int32), ("flags", ctypes.c_int32)]


class ChainOpts(ctypes.Structure):
    """``mxfp4_chain_opts`` of the header."""
    _fields_ = [("wait_us", ctypes.c_int64), ("phantom_workgroups", ctypes.c_int32), ("mode", ctypes.c_int32)]


class KvCacheDesc(ctypes.Structure):
    """``mxfp4_kv_cache`` of the header, field for field (as the four below it)."""
    _fields_ = [("kq", ctypes.c_void_p), ("ks", ctypes.c_void_p), ("vq", ctypes.c_void_p), ("vs", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("page_stride_q", ctypes.c_int64), ("page_stride_s", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("page", ctypes.c_int32), ("dim", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class KvRowsDesc(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("ldt", ctypes.c_int64), ("width", ctypes.c_int64), ("lens", ctypes.c_void_p),
                ("starts", ctypes.c_void_p), ("rows", ctypes.c_int64), ("tokens", ctypes.c_int64)]


class KvRopeDesc(ctypes.Structure):
    _fields_ = [("cos_f32", ctypes.c_void_p), ("sin_f32", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("length", ctypes.c_int64), ("dim", ctypes.c_int64)]


class KvTensorDesc(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class KvAttentionArgs(ctypes.Structure):
    _fields_ = [("q", KvTensorDesc), ("out", KvTensorDesc), ("lse_f32", ctypes.c_void_p), ("tree", ctypes.c_void_p),
                ("q_heads", ctypes.c_int64), ("window", ctypes.c_int64), ("scale", ctypes.c_float), ("causal", ctypes.c_int32)]


class KvPoolDesc(ctypes.Structure):
    _fields_ = [("refs", ctypes.c_void_p), ("free_bits", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page", ctypes.c_int64),
                ("table", ctypes.c_void_p), ("ldt", ctypes.c_int64), ("width", ctypes.c_int64), ("rows", ctypes.c_int64),
                ("lens", ctypes.c_void_p)]


KV_COUNTERS = 16384
CHAIN_STATUS_OFFSET = 4224
CHAIN_AUTO, CHAIN_PERSISTENT, CHAIN_SEPARATE = 0, 1, 2


class Mxfp4Error(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("mxfp4 error %d: %s" % (code, text))
        self.code = code


def load() -> ctypes.CDLL:
    """Load the HIP library (torch first, so that both share one HIP runtime)."""
    global _lib, _product, _verify, _cast, _kv
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s is missing: build it with `python -m paper_2503_13565_amd.build`; "
            "there is no fallback path" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    lib.mxfp4_direct_cast.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    lib.mxfp4_direct_cast_bits.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    lib.mxfp4_direct_cast_bits.restype = i32
    lib.mxfp4_dequant.argtypes = [vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_dequant_hwcvt.argtypes = [vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_woq_gemm.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_woq_gemm_path.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, i32, vp]
    lib.mxfp4_woq_gemm_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mxfp4_woq_gemm_workspace_bytes.restype = sz
    lib.mxfp4_woq_gemm_ws.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp, sz, i32, vp]
    lib.mxfp4_woq_gemm_ws.restype = i32
    lib.mxfp4_woq_gemm_argmax_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mxfp4_woq_gemm_argmax_workspace_bytes.restype = sz
    lib.mxfp4_woq_gemm_argmax.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.mxfp4_woq_gemm_argmax_path.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, sz, i32, vp]
    lib.mxfp4_bf16_gemm.argtypes = [vp, i64, i64, vp, i64, i64, i64, vp, i64, vp]
    lib.mxfp4_bf16_gemm.restype = i32
    lib.mxfp4_bf16_gemm_argmax_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mxfp4_bf16_gemm_argmax_workspace_bytes.restype = sz
    lib.mxfp4_bf16_gemm_argmax.argtypes = [vp, i64, i64, vp, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.mxfp4_bf16_gemm_argmax.restype = i32
    lib.mxfp4_woq_gemm_verify.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.mxfp4_woq_gemm_verify.restype = i32
    lib.mxfp4_bf16_gemm_verify.argtypes = [vp, i64, i64, vp, i64, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.mxfp4_bf16_gemm_verify.restype = i32
    for name in ("mxfp4_e4m3_direct_cast", "mxfp4_e4m3_direct_cast_bits"):
        getattr(lib, name).argtypes = [vp, i64, i64, i64, vp, vp, vp]
        getattr(lib, name).restype = i32
    lib.mxfp4_e4m3_dequant.argtypes = [vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_e4m3_dequant.restype = i32
    lib.mxfp4_e4m3_woq_gemm.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_e4m3_woq_gemm.restype = i32
    lib.mxfp4_e4m3_woq_gemm_argmax.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.mxfp4_e4m3_woq_gemm_argmax.restype = i32
    for name in ("mxfp4_e2m3_direct_cast", "mxfp4_e2m3_direct_cast_bits"):
        getattr(lib, name).argtypes = [vp, i64, i64, i64, vp, vp, vp]
        getattr(lib, name).restype = i32
    lib.mxfp4_e2m3_dequant.argtypes = [vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_e2m3_dequant.restype = i32
    lib.mxfp4_e2m3_woq_gemm.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_e2m3_woq_gemm.restype = i32
    lib.mxfp4_e2m3_woq_gemm_argmax.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.mxfp4_e2m3_woq_gemm_argmax.restype = i32
    lib.mxfp4_woq_gemm_t_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mxfp4_woq_gemm_t_workspace_bytes.restype = sz
    lib.mxfp4_woq_gemm_t.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp, sz, vp]
    lib.mxfp4_woq_gemm_t.restype = i32
    lib.mxfp4_fmt_block_bytes.argtypes = [i32]
    lib.mxfp4_fmt_block_bytes.restype = i32
    for name in ("mxfp4_fmt_direct_cast", "mxfp4_fmt_direct_cast_bits"):
        getattr(lib, name).argtypes = [i32, vp, i64, i64, i64, vp, vp, vp]
        getattr(lib, name).restype = i32
    lib.mxfp4_fmt_dequant.argtypes = [i32, vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_fmt_dequant.restype = i32
    lib.mxfp4_fmt_woq_gemm.argtypes = [i32, vp, i64, i64, vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_fmt_woq_gemm.restype = i32
    lib.mxfp4_fmt_woq_gemm_argmax.argtypes = [i32, vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.mxfp4_fmt_woq_gemm_argmax.restype = i32
    lib.mxfp4_woq_gemm_fused.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i32, vp, i64, vp, i64, vp, sz, i32, vp]
    lib.mxfp4_woq_gemm_fused.restype = i32
    lib.mxfp4_tile_repack_q_bytes.argtypes = [i64, i64]
    lib.mxfp4_tile_repack_q_bytes.restype = sz
    lib.mxfp4_tile_repack_s_bytes.argtypes = [i64, i64]
    lib.mxfp4_tile_repack_s_bytes.restype = sz
    lib.mxfp4_tile_repack.argtypes = [vp, vp, i64, i64, vp, vp, vp]
    lib.mxfp4_tile_repack.restype = i32
    lib.mxfp4_woq_gemm_tiled.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp]
    lib.mxfp4_woq_gemm_tiled.restype = i32
    lib.mxfp4_woq_gemm_tiled_ws.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i64, vp, sz, vp]
    lib.mxfp4_woq_gemm_tiled_ws.restype = i32
    lib.mxfp4_woq_gemm_tiled_argmax.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.mxfp4_woq_gemm_tiled_argmax.restype = i32
    lib.mxfp4_woq_gemm_tiled_verify.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.mxfp4_woq_gemm_tiled_verify.restype = i32
    lib.mxfp4_woq_gemm_tiled_fused.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, i32, vp, i64, vp, i64, vp]
    lib.mxfp4_woq_gemm_tiled_fused.restype = i32
    lib.mxfp4_woq_gemm_grouped_workspace_bytes.argtypes = [ctypes.POINTER(GemmDesc), i64]
    lib.mxfp4_woq_gemm_grouped_workspace_bytes.restype = sz
    lib.mxfp4_woq_gemm_grouped.argtypes = [ctypes.POINTER(GemmDesc), i64, vp, sz, vp]
    lib.mxfp4_woq_gemm_grouped.restype = i32
    lib.mxfp4_woq_gemm_argmax_noalloc_max_bytes.argtypes = []
    lib.mxfp4_woq_gemm_argmax_noalloc_max_bytes.restype = sz
    lib.mxfp4_woq_gemm_argmax_noalloc.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, vp]
    lib.mxfp4_woq_gemm_argmax_noalloc.restype = i32
    lib.mxfp4_woq_gemm_chain_workspace_bytes.argtypes = []
    lib.mxfp4_woq_gemm_chain_workspace_bytes.restype = sz
    lib.mxfp4_woq_gemm_chain_init.argtypes = [vp, sz, vp]
    lib.mxfp4_woq_gemm_chain_init.restype = i32
    lib.mxfp4_woq_gemm_chain.argtypes = [ctypes.POINTER(GemmDesc), i64, vp, sz, ctypes.POINTER(ChainOpts), vp]
    lib.mxfp4_woq_gemm_chain.restype = i32
    ref = ctypes.POINTER
    lib.mxfp4_kv_append.argtypes = [ref(KvCacheDesc), ref(KvRowsDesc), ref(KvTensorDesc), ref(KvTensorDesc), ref(KvTensorDesc),
                                    ref(KvTensorDesc), i64, ref(KvRopeDesc), vp]
    lib.mxfp4_kv_read.argtypes = [ref(KvCacheDesc), ref(KvRowsDesc), ref(KvTensorDesc), ref(KvTensorDesc), vp]
    lib.mxfp4_kv_attention_workspace_bytes.argtypes = [ref(KvCacheDesc), ref(KvRowsDesc), i64]
    lib.mxfp4_kv_attention_workspace_bytes.restype = sz
    lib.mxfp4_kv_attention.argtypes = [ref(KvCacheDesc), ref(KvRowsDesc), ref(KvAttentionArgs), vp, sz, vp]
    lib.mxfp4_kv_fork.argtypes = [ref(KvPoolDesc), vp, vp, i64, vp]
    lib.mxfp4_kv_extend.argtypes = [ref(KvPoolDesc), ref(KvCacheDesc), vp, vp, i64, vp, vp, vp]
    lib.mxfp4_kv_release.argtypes = [ref(KvPoolDesc), vp, vp, i64, vp]
    lib.mxfp4_kv_compact.argtypes = [ref(KvCacheDesc), vp, i64, i64, vp, vp, i64, vp, i64, vp]
    lib.mxfp4_kv_copy_pages.argtypes = [ref(KvCacheDesc), vp, vp, i64, vp]
    for name in ("append", "read", "attention", "fork", "extend", "release", "compact", "copy_pages"):
        getattr(lib, "mxfp4_kv_" + name).restype = i32
    lib.mxfp4_diag_stream_read.argtypes = [vp, sz, vp, vp]
    lib.mxfp4_diag_stream_copy.argtypes = [vp, vp, sz, vp]
    for name in ("mxfp4_direct_cast", "mxfp4_direct_cast_bits", "mxfp4_dequant", "mxfp4_dequant_hwcvt", "mxfp4_woq_gemm",
                 "mxfp4_woq_gemm_path", "mxfp4_woq_gemm_argmax", "mxfp4_woq_gemm_argmax_path",
                 "mxfp4_diag_stream_read", "mxfp4_diag_stream_copy"):
        getattr(lib, name).restype = i32
    lib.mxfp4_last_error.restype = ctypes.c_char_p
    lib.mxfp4_version.restype = ctypes.c_char_p
    _product, _verify, _cast, _kv = _host_calls()
    _lib = lib
    return lib


def _host_calls():
    """The calls of the extension module.  Without it, or with one that was built for another torch, every call takes
    the checks here, which reach the same kernels with more host time."""
    try:
        from . import _host
        if _host.torch_version != str(torch.__version__):
            raise ImportError("built for torch %s" % _host.torch_version)
    except ImportError as e:
        warnings.warn("the extension module _host cannot be used (%s): calls go through ctypes, which takes more host time; "
                      "build it with `python -m paper_2503_13565_amd.build`" % e, RuntimeWarning, stacklevel=3)
        return (*(lambda *args: None,) * 3, _Kv)
    _host.on_failure(_check)

    class kv(_Kv):
        append, read, attention, pages, compact = _host.kv_append, _host.kv_read, _host.kv_attention, _host.kv_pages, _host.kv_compact
    return _host.product, _host.verify, _host.cast, kv


def _check(rc: int) -> None:
    if rc != 0:
        raise Mxfp4Error(rc, load().mxfp4_last_error().decode())


# What surrounds a call costs more host time than the call's checks and as much as its launch, and most of the
# products here are shorter on the device than that.  So addresses go to ctypes as plain integers, the stream is
# asked for as the integer it is, and the device is switched only where another one is current (one product
# 10.9 -> 6.9 us of host time; through the extension module 3.5).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_stay = contextlib.nullcontext()


def _on(device: torch.device):
    """Context in which ``device`` is the current device."""
    return _stay if device.index == _current_device() else torch.cuda.device(device)


def _stream() -> int:
    """The current stream of the current device."""
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(_current_device())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor) -> None:
    if not t.is_cuda:
        raise ValueError("tensor must live in GPU memory")


def version() -> str:
    return load().mxfp4_version().decode()


def mxfp4_direct_cast(w: torch.Tensor, q: Optional[torch.Tensor] = None,
                      s: Optional[torch.Tensor] = None, integer_rule: bool = False
                      ) -> Tuple[torch.Tensor, torch.Tensor]:
    """BF16 ``[N,K]`` (last dim contiguous) -> (q uint8 ``[N,K/2]``, s uint8 ``[N,K/32]``).
    ``integer_rule`` calls ``mxfp4_direct_cast_bits``."""
    if q is None and s is None and not integer_rule:
        pair = _cast(w)
        if pair is not None:
            return pair
    _dev(w)
    if w.dtype != torch.bfloat16 or w.dim() != 2 or w.stride(1) != 1:
        raise ValueError("w must be a 2-D BF16 tensor with a contiguous last dimension")
    n, k = w.shape
    if q is None:
        q = torch.empty((n, k // 2), dtype=torch.uint8, device=w.device)
    if s is None:
        s = torch.empty((n, k // 32), dtype=torch.uint8, device=w.device)
    ldw = w.stride(0) if n > 1 else max(k, 1)
    with _on(w.device):
        fn = load().mxfp4_direct_cast_bits if integer_rule else load().mxfp4_direct_cast
        _check(fn(_ptr(w), n, k, ldw, _ptr(q), _ptr(s), _stream()))
    return q, s


def mxfp4_dequant(q: torch.Tensor, s: torch.Tensor, hw_convert: bool = False) -> torch.Tensor:
    _dev(q)
    n, k = q.shape[0], q.shape[1] * 2
    w = torch.empty((n, k), dtype=torch.bfloat16, device=q.device)
    fn = load().mxfp4_dequant_hwcvt if hw_convert else load().mxfp4_dequant
    with _on(q.device):
        _check(fn(_ptr(q), _ptr(s), n, k, _ptr(w), k, _stream()))
    return w


def _gemm_shapes(x, q, s):
    _dev(x)
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D BF16 tensor with a contiguous last dimension")
    if q.dtype != torch.uint8 or s.dtype != torch.uint8 or not q.is_contiguous() or not s.is_contiguous():
        raise ValueError("q and s must be contiguous uint8 tensors")
    m, k = x.shape
    n = q.shape[0]
    if q.shape[1] * 2 != k or tuple(s.shape) != (n, k // 32):
        raise ValueError("shape mismatch: x %r q %r s %r" % (tuple(x.shape), tuple(q.shape), tuple(s.shape)))
    ldx = x.stride(0) if m > 1 else k
    return m, n, k, ldx


def mxfp4_woq_gemm(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor, y: Optional[torch.Tensor] = None,
                   path: int = PATH_AUTO, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y ``[M,N]`` BF16 = x ``[M,K]`` BF16 times dequant(q, s)^T.  With ``workspace`` (uint8, at least
    ``mxfp4_woq_gemm_workspace_bytes``) the call goes through ``mxfp4_woq_gemm_ws``."""
    if y is None:
        y = _product(_MX, x, q, s, 0, 0, False, None, 0, None, path, workspace)
        if y is not None:
            return y
    m, n, k, ldx = _gemm_shapes(x, q, s)
    if y is None:
        y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    ldy = y.stride(0) if m > 1 else n
    with _on(x.device):
        if workspace is None:
            _check(load().mxfp4_woq_gemm_path(_ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(y), ldy, path,
                                             _stream()))
        else:
            _check(load().mxfp4_woq_gemm_ws(_ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(y), ldy,
                                           _ptr(workspace), workspace.numel() * workspace.element_size(),
                                           path, _stream()))
    return y


def mxfp4_woq_gemm_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(load().mxfp4_woq_gemm_workspace_bytes(m, n, k))


def mxfp4_woq_gemm_argmax_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(load().mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k))


def mxfp4_woq_gemm_argmax(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor,
                          workspace: Optional[torch.Tensor] = None, path: int = PATH_AUTO,
                          out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                          ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Row-wise (argmax int32 ``[M]``, max float32 ``[M]``) of x times dequant(q, s)^T."""
    m, n, k, ldx = _gemm_shapes(x, q, s)
    need = mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k)
    if workspace is None:
        workspace = torch.empty((need,), dtype=torch.uint8, device=x.device)
    if out is None:
        idx = torch.empty((m,), dtype=torch.int32, device=x.device)
        val = torch.empty((m,), dtype=torch.float32, device=x.device)
    else:
        idx, val = out
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_argmax_path(_ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(idx), _ptr(val),
                                                _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                path, _stream()))
    return idx, val


def mxfp4_woq_gemm_argmax_noalloc(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor,
                                  out: Tuple[torch.Tensor, torch.Tensor]) -> Tuple[torch.Tensor, torch.Tensor]:
    """The fused pick on the library's own scratch: nothing is allocated here either, so the caller
    brings ``out = (idx int32 [M], val float32 [M])``."""
    m, n, k, ldx = _gemm_shapes(x, q, s)
    idx, val = out
    if (idx.dtype != torch.int32 or val.dtype != torch.float32 or idx.shape != (m,) or val.shape != (m,)
            or not idx.is_contiguous() or not val.is_contiguous()):
        raise ValueError("out must be (int32 [M], float32 [M]), contiguous")
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_argmax_noalloc(_ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(idx), _ptr(val),
                                                    _stream()))
    return idx, val


def _bf16_shapes(x, w):
    _dev(x)
    for t, what in ((x, "x"), (w, "w")):
        if t.dtype != torch.bfloat16 or t.dim() != 2 or t.stride(1) != 1:
            raise ValueError("%s must be a 2-D BF16 tensor with a contiguous last dimension" % what)
    m, k = x.shape
    n = w.shape[0]
    if w.shape[1] != k:
        raise ValueError("shape mismatch: x %r w %r" % (tuple(x.shape), tuple(w.shape)))
    return m, n, k, (x.stride(0) if m > 1 else k), (w.stride(0) if n > 1 else k)


def mxfp4_bf16_gemm(x: torch.Tensor, w: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y ``[M,N]`` BF16 = x ``[M,K]`` BF16 times w ``[N,K]``^T with unquantised BF16 weights."""
    if y is None:
        y = _product(_BF16, x, w, None, 0, 0, False, None, 0, None, 0, None)
        if y is not None:
            return y
    m, n, k, ldx, ldw = _bf16_shapes(x, w)
    if y is None:
        y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    with _on(x.device):
        _check(load().mxfp4_bf16_gemm(_ptr(x), m, ldx, _ptr(w), n, k, ldw, _ptr(y),
                                     y.stride(0) if m > 1 else n, _stream()))
    return y


def mxfp4_bf16_gemm_argmax_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(load().mxfp4_bf16_gemm_argmax_workspace_bytes(m, n, k))


def mxfp4_bf16_gemm_argmax(x: torch.Tensor, w: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                           out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                           ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Row-wise (argmax int32 ``[M]``, max float32 ``[M]``) of x times w^T."""
    m, n, k, ldx, ldw = _bf16_shapes(x, w)
    if workspace is None:
        workspace = torch.empty((mxfp4_bf16_gemm_argmax_workspace_bytes(m, n, k),), dtype=torch.uint8,
                                device=x.device)
    if out is None:
        idx = torch.empty((m,), dtype=torch.int32, device=x.device)
        val = torch.empty((m,), dtype=torch.float32, device=x.device)
    else:
        idx, val = out
    with _on(x.device):
        _check(load().mxfp4_bf16_gemm_argmax(_ptr(x), m, ldx, _ptr(w), n, k, ldw, _ptr(idx), _ptr(val),
                                            _ptr(workspace), workspace.numel() * workspace.element_size(),
                                            _stream()))
    return idx, val


def _verify_buffers(x, m, draft, need, workspace):
    if draft is not None and (draft.dtype != torch.int32 or draft.numel() != m - 1 or not draft.is_contiguous()):
        raise ValueError("draft must hold M - 1 contiguous int32 tokens")
    if workspace is None:
        workspace = torch.empty((need,), dtype=torch.uint8, device=x.device)
    accept = torch.empty((2,), dtype=torch.int32, device=x.device)
    idx = torch.empty((m,), dtype=torch.int32, device=x.device)
    val = torch.empty((m,), dtype=torch.float32, device=x.device)
    return workspace, accept, idx, val


def mxfp4_woq_gemm_verify(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor, draft: Optional[torch.Tensor],
                          workspace: Optional[torch.Tensor] = None):
    """(accept int32 ``[2]`` = (G, next token), argmax int32 ``[M]``, max float32 ``[M]``)."""
    got = _verify(_MX, x, q, s, 0, 0, draft, workspace)
    if got is not None:
        return got
    m, n, k, ldx = _gemm_shapes(x, q, s)
    workspace, accept, idx, val = _verify_buffers(x, m, draft, mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k),
                                                  workspace)
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_verify(_ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(draft), _ptr(accept),
                                           _ptr(idx), _ptr(val), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), _stream()))
    return accept, idx, val


def mxfp4_e4m3_direct_cast(w: torch.Tensor, integer_rule: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """BF16 ``[N, K]`` -> (``q8 [N, K]`` E4M3 bytes, ``s [N, K/32]`` E8M0 scale bytes)."""
    _dev(w)
    if w.dtype != torch.bfloat16 or w.dim() != 2 or w.stride(1) != 1:
        raise ValueError("w must be a 2-D BF16 tensor with a contiguous last dimension")
    n, k = w.shape
    q8 = torch.empty((n, k), dtype=torch.uint8, device=w.device)
    s = torch.empty((n, k // 32), dtype=torch.uint8, device=w.device)
    fn = load().mxfp4_e4m3_direct_cast_bits if integer_rule else load().mxfp4_e4m3_direct_cast
    with _on(w.device):
        _check(fn(_ptr(w), n, k, w.stride(0) if n > 1 else k, _ptr(q8), _ptr(s), _stream()))
    return q8, s


def mxfp4_e4m3_dequant(q8: torch.Tensor, s: torch.Tensor) -> torch.Tensor:
    _dev(q8)
    n, k = q8.shape
    w = torch.empty((n, k), dtype=torch.bfloat16, device=q8.device)
    with _on(q8.device):
        _check(load().mxfp4_e4m3_dequant(_ptr(q8), _ptr(s), n, k, _ptr(w), k, _stream()))
    return w


def _e4m3_shapes(x, q8, s):
    _dev(x)
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D BF16 tensor with a contiguous last dimension")
    if q8.dtype != torch.uint8 or s.dtype != torch.uint8 or not q8.is_contiguous() or not s.is_contiguous():
        raise ValueError("q8 and s must be contiguous uint8 tensors")
    m, k = x.shape
    n = q8.shape[0]
    if q8.shape[1] != k or tuple(s.shape) != (n, k // 32):
        raise ValueError("shape mismatch: x %r q8 %r s %r" % (tuple(x.shape), tuple(q8.shape), tuple(s.shape)))
    return m, n, k, (x.stride(0) if m > 1 else k)


def mxfp4_e4m3_woq_gemm(x: torch.Tensor, q8: torch.Tensor, s: torch.Tensor,
                        y: Optional[torch.Tensor] = None) -> torch.Tensor:
    if y is None:
        y = _product(_E4M3, x, q8, s, 0, 0, False, None, 0, None, 0, None)
        if y is not None:
            return y
    m, n, k, ldx = _e4m3_shapes(x, q8, s)
    if y is None:
        y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    with _on(x.device):
        _check(load().mxfp4_e4m3_woq_gemm(_ptr(x), m, ldx, _ptr(q8), _ptr(s), n, k, _ptr(y),
                                         y.stride(0) if m > 1 else n, _stream()))
    return y


def mxfp4_e4m3_woq_gemm_argmax(x: torch.Tensor, q8: torch.Tensor, s: torch.Tensor,
                               workspace: Optional[torch.Tensor] = None,
                               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                               ) -> Tuple[torch.Tensor, torch.Tensor]:
    m, n, k, ldx = _e4m3_shapes(x, q8, s)
    if workspace is None:
        workspace = torch.empty((mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k),), dtype=torch.uint8,
                                device=x.device)
    if out is None:
        idx = torch.empty((m,), dtype=torch.int32, device=x.device)
        val = torch.empty((m,), dtype=torch.float32, device=x.device)
    else:
        idx, val = out
    with _on(x.device):
        _check(load().mxfp4_e4m3_woq_gemm_argmax(_ptr(x), m, ldx, _ptr(q8), _ptr(s), n, k, _ptr(idx), _ptr(val),
                                                _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                _stream()))
    return idx, val


def mxfp4_e2m3_direct_cast(w: torch.Tensor, integer_rule: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """BF16 ``[N, K]`` -> (``q6 [N, K/32*24]`` packed E2M3 codes, ``s [N, K/32]`` E8M0 scale bytes)."""
    _dev(w)
    if w.dtype != torch.bfloat16 or w.dim() != 2 or w.stride(1) != 1:
        raise ValueError("w must be a 2-D BF16 tensor with a contiguous last dimension")
    n, k = w.shape
    q6 = torch.empty((n, k // 32 * 24), dtype=torch.uint8, device=w.device)
    s = torch.empty((n, k // 32), dtype=torch.uint8, device=w.device)
    fn = load().mxfp4_e2m3_direct_cast_bits if integer_rule else load().mxfp4_e2m3_direct_cast
    with _on(w.device):
        _check(fn(_ptr(w), n, k, w.stride(0) if n > 1 else k, _ptr(q6), _ptr(s), _stream()))
    return q6, s


def mxfp4_e2m3_dequant(q6: torch.Tensor, s: torch.Tensor) -> torch.Tensor:
    _dev(q6)
    n, k = s.shape[0], s.shape[1] * 32
    w = torch.empty((n, k), dtype=torch.bfloat16, device=q6.device)
    with _on(q6.device):
        _check(load().mxfp4_e2m3_dequant(_ptr(q6), _ptr(s), n, k, _ptr(w), k, _stream()))
    return w


def _e2m3_shapes(x, q6, s):
    _dev(x)
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D BF16 tensor with a contiguous last dimension")
    if q6.dtype != torch.uint8 or s.dtype != torch.uint8 or not q6.is_contiguous() or not s.is_contiguous():
        raise ValueError("q6 and s must be contiguous uint8 tensors")
    m, k = x.shape
    n = q6.shape[0]
    if q6.shape[1] != k // 32 * 24 or tuple(s.shape) != (n, k // 32):
        raise ValueError("shape mismatch: x %r q6 %r s %r" % (tuple(x.shape), tuple(q6.shape), tuple(s.shape)))
    return m, n, k, (x.stride(0) if m > 1 else k)


def mxfp4_e2m3_woq_gemm(x: torch.Tensor, q6: torch.Tensor, s: torch.Tensor,
                        y: Optional[torch.Tensor] = None) -> torch.Tensor:
    if y is None:
        y = _product(_E2M3, x, q6, s, 0, 0, False, None, 0, None, 0, None)
        if y is not None:
            return y
    m, n, k, ldx = _e2m3_shapes(x, q6, s)
    if y is None:
        y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    with _on(x.device):
        _check(load().mxfp4_e2m3_woq_gemm(_ptr(x), m, ldx, _ptr(q6), _ptr(s), n, k, _ptr(y),
                                         y.stride(0) if m > 1 else n, _stream()))
    return y


def mxfp4_e2m3_woq_gemm_argmax(x: torch.Tensor, q6: torch.Tensor, s: torch.Tensor,
                               workspace: Optional[torch.Tensor] = None,
                               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                               ) -> Tuple[torch.Tensor, torch.Tensor]:
    m, n, k, ldx = _e2m3_shapes(x, q6, s)
    if workspace is None:
        workspace = torch.empty((mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k),), dtype=torch.uint8,
                                device=x.device)
    if out is None:
        idx = torch.empty((m,), dtype=torch.int32, device=x.device)
        val = torch.empty((m,), dtype=torch.float32, device=x.device)
    else:
        idx, val = out
    with _on(x.device):
        _check(load().mxfp4_e2m3_woq_gemm_argmax(_ptr(x), m, ldx, _ptr(q6), _ptr(s), n, k, _ptr(idx), _ptr(val),
                                                _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                _stream()))
    return idx, val


def mxfp4_woq_gemm_t_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(load().mxfp4_woq_gemm_t_workspace_bytes(m, n, k))


def mxfp4_woq_gemm_t(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor, y: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``y[M, K] = x[M, N] @ dequant(q, s)[N, K]``: the product along the rows of the stored tensor."""
    _dev(x)
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D BF16 tensor with a contiguous last dimension")
    if q.dtype != torch.uint8 or s.dtype != torch.uint8 or not q.is_contiguous() or not s.is_contiguous():
        raise ValueError("q and s must be contiguous uint8 tensors")
    m, n = x.shape
    k = q.shape[1] * 2
    if q.shape[0] != n or tuple(s.shape) != (n, k // 32):
        raise ValueError("shape mismatch: x %r q %r s %r" % (tuple(x.shape), tuple(q.shape), tuple(s.shape)))
    if y is None:
        y = torch.empty((m, k), dtype=torch.bfloat16, device=x.device)
    if workspace is None:
        workspace = torch.empty((max(mxfp4_woq_gemm_t_workspace_bytes(m, n, k), 4),), dtype=torch.uint8,
                                device=x.device)
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_t(_ptr(x), m, x.stride(0) if m > 1 else n, _ptr(q), _ptr(s), n, k, _ptr(y),
                                      y.stride(0) if m > 1 else k, _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream()))
    return y


FMT_E5M2, FMT_E3M2, FMT_T2 = 1, 2, 3


def mxfp4_fmt_block_bytes(fmt: int) -> int:
    """Bytes of one 32-element block of the format (32, 24, 8); 0 for an unknown id."""
    return int(load().mxfp4_fmt_block_bytes(fmt))


def mxfp4_fmt_direct_cast(fmt: int, w: torch.Tensor, integer_rule: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """BF16 ``[N, K]`` -> (``q [N, K/32 * block_bytes]`` packed codes, ``s [N, K/32]`` E8M0 scale bytes)."""
    _dev(w)
    if w.dtype != torch.bfloat16 or w.dim() != 2 or w.stride(1) != 1:
        raise ValueError("w must be a 2-D BF16 tensor with a contiguous last dimension")
    n, k = w.shape
    q = torch.empty((n, k // 32 * max(mxfp4_fmt_block_bytes(fmt), 1)), dtype=torch.uint8, device=w.device)
    s = torch.empty((n, k // 32), dtype=torch.uint8, device=w.device)
    fn = load().mxfp4_fmt_direct_cast_bits if integer_rule else load().mxfp4_fmt_direct_cast
    with _on(w.device):
        _check(fn(fmt, _ptr(w), n, k, w.stride(0) if n > 1 else k, _ptr(q), _ptr(s), _stream()))
    return q, s


def mxfp4_fmt_dequant(fmt: int, q: torch.Tensor, s: torch.Tensor) -> torch.Tensor:
    _dev(q)
    n, k = s.shape[0], s.shape[1] * 32
    w = torch.empty((n, k), dtype=torch.bfloat16, device=q.device)
    with _on(q.device):
        _check(load().mxfp4_fmt_dequant(fmt, _ptr(q), _ptr(s), n, k, _ptr(w), k, _stream()))
    return w


def _fmt_shapes(fmt, x, q, s):
    _dev(x)
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D BF16 tensor with a contiguous last dimension")
    if q.dtype != torch.uint8 or s.dtype != torch.uint8 or not q.is_contiguous() or not s.is_contiguous():
        raise ValueError("q and s must be contiguous uint8 tensors")
    m, k = x.shape
    n = q.shape[0]
    bb = mxfp4_fmt_block_bytes(fmt)
    if bb and (q.shape[1] != k // 32 * bb or tuple(s.shape) != (n, k // 32)):
        raise ValueError("shape mismatch: x %r q %r s %r" % (tuple(x.shape), tuple(q.shape), tuple(s.shape)))
    return m, n, k, (x.stride(0) if m > 1 else k)


def mxfp4_fmt_woq_gemm(fmt: int, x: torch.Tensor, q: torch.Tensor, s: torch.Tensor,
                       y: Optional[torch.Tensor] = None) -> torch.Tensor:
    if y is None and type(fmt) is int and FMT_E5M2 <= fmt <= FMT_T2:
        y = _product(_FMT + fmt, x, q, s, 0, 0, False, None, 0, None, 0, None)
        if y is not None:
            return y
    m, n, k, ldx = _fmt_shapes(fmt, x, q, s)
    if y is None:
        y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    with _on(x.device):
        _check(load().mxfp4_fmt_woq_gemm(fmt, _ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(y),
                                        y.stride(0) if m > 1 else n, _stream()))
    return y


def mxfp4_fmt_woq_gemm_argmax(fmt: int, x: torch.Tensor, q: torch.Tensor, s: torch.Tensor,
                              workspace: Optional[torch.Tensor] = None,
                              out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                              ) -> Tuple[torch.Tensor, torch.Tensor]:
    m, n, k, ldx = _fmt_shapes(fmt, x, q, s)
    if workspace is None:
        workspace = torch.empty((mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k),), dtype=torch.uint8,
                                device=x.device)
    if out is None:
        idx = torch.empty((m,), dtype=torch.int32, device=x.device)
        val = torch.empty((m,), dtype=torch.float32, device=x.device)
    else:
        idx, val = out
    with _on(x.device):
        _check(load().mxfp4_fmt_woq_gemm_argmax(fmt, _ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(idx), _ptr(val),
                                               _ptr(workspace), workspace.numel() * workspace.element_size(),
                                               _stream()))
    return idx, val


ACT_NONE, ACT_SWIGLU = 0, 1


def mxfp4_woq_gemm_fused(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor, bias: Optional[torch.Tensor] = None,
                         act: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
                         y: Optional[torch.Tensor] = None, path: int = PATH_AUTO,
                         workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The product with bias, gate and residual add fused; ``residual`` may be ``y`` itself."""
    if y is None:
        y = _product(_MX, x, q, s, 0, 0, True, bias, act, residual, path, workspace)
        if y is not None:
            return y
    m, n, k, ldx = _gemm_shapes(x, q, s)
    c = n // 2 if act == ACT_SWIGLU else n
    if bias is not None and (bias.dtype != torch.bfloat16 or bias.dim() != 1 or bias.shape[0] != n
                             or not bias.is_contiguous() or bias.device != x.device):
        raise ValueError("bias must be a contiguous BF16 tensor [N] on the device of x")
    if residual is not None and (residual.dtype != torch.bfloat16 or residual.dim() != 2
                                 or residual.shape != (m, c) or residual.stride(1) != 1
                                 or residual.device != x.device):
        raise ValueError("residual must be a BF16 tensor [M, %d] with a contiguous last dimension" % c)
    if y is None:
        y = torch.empty((m, c), dtype=torch.bfloat16, device=x.device)
    ldy = y.stride(0) if m > 1 else c
    ldr = (residual.stride(0) if m > 1 else c) if residual is not None else 0
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_fused(
            _ptr(x), m, ldx, _ptr(q), _ptr(s), n, k, _ptr(bias), act, _ptr(residual), ldr, _ptr(y), ldy,
            _ptr(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0, path,
            _stream()))
    return y


DESC_TILED = 1
DESC_INDEPENDENT = 2


class GemmGroup:
    """A fixed sequence of products (``mxfp4_woq_gemm_grouped``): the descriptor array is built once,
    ``run()`` is one library call.  ``items``: dicts with ``x``, ``q``, ``s`` and optionally ``bias``,
    ``act``, ``residual``, ``y`` (allocated when missing), as for ``mxfp4_woq_gemm_fused``; or with
    ``argmax=True`` (optionally ``out=(idx int32 [M], val float32 [M])``) for the fused pick, whose
    entry in ``ys`` is the ``(idx, val)`` pair.  The tensors are kept alive by the group; ``ys`` lists
    the outputs in order.  An item with ``w`` (a ``TiledWeights``) in place of ``q`` and ``s`` runs on
    the tile-major copy.  ``independent=True`` on an item sets ``MXFP4_DESC_INDEPENDENT``: neighbouring
    items that carry it and do not read each other's outputs may share one launch.
    ``chained=True``: ``run()`` is ``mxfp4_woq_gemm_chain`` (a dependent sequence of one-token
    products on canonical tensors, ``mode`` = ``CHAIN_AUTO``, ``CHAIN_PERSISTENT`` or
    ``CHAIN_SEPARATE``); the group then owns a chain workspace, prepared once, and
    ``chain_status()`` reads its status word (synchronises)."""

    def __init__(self, items, chained: bool = False, wait_us: int = 0, phantom_workgroups: int = 0,
                 mode: int = 0):
        self._keep, self.ys = [], []
        self._descs = (GemmDesc * max(1, len(items)))()
        self.count = len(items)
        for d, it in zip(self._descs, items):
            x = it["x"]
            bias, residual, act = it.get("bias"), it.get("residual"), int(it.get("act", ACT_NONE))
            if "w" in it:                                  # TiledWeights in place of (q, s)
                q, s = it["w"].q, it["w"].s
                m, n, k, ldx = _tiled_shapes(x, it["w"])
                d.flags = DESC_TILED
            else:
                q, s = it["q"], it["s"]
                m, n, k, ldx = _gemm_shapes(x, q, s)
                d.flags = 0
            if it.get("independent"):
                d.flags |= DESC_INDEPENDENT
            d.x_bf16, d.M, d.ldx = x.data_ptr(), m, ldx
            d.q_packed, d.scales_e8m0, d.N, d.K = q.data_ptr(), s.data_ptr(), n, k
            d.act = act
            if it.get("argmax"):
                idx, val = it.get("out") or (torch.empty((m,), dtype=torch.int32, device=x.device),
                                             torch.empty((m,), dtype=torch.float32, device=x.device))
                if (idx.dtype != torch.int32 or val.dtype != torch.float32 or idx.shape != (m,) or val.shape != (m,)
                        or not idx.is_contiguous() or not val.is_contiguous()):
                    raise ValueError("out must be (int32 [M], float32 [M]), contiguous")
                d.argmax_out, d.max_out = idx.data_ptr(), val.data_ptr()
                self._keep.append((x, q, s, idx, val))
                self.ys.append((idx, val))
                continue
            c = n // 2 if act == ACT_SWIGLU else n
            y = it.get("y")
            if y is None:
                y = torch.empty((m, c), dtype=torch.bfloat16, device=x.device)
            if y.dtype != torch.bfloat16 or y.dim() != 2 or y.shape != (m, c) or y.stride(1) != 1:
                raise ValueError("y must be a BF16 tensor [M, %d] with a contiguous last dimension" % c)
            if bias is not None and (bias.dtype != torch.bfloat16 or bias.shape != (n,) or not bias.is_contiguous()):
                raise ValueError("bias must be a contiguous BF16 tensor [N]")
            if residual is not None and (residual.dtype != torch.bfloat16 or residual.shape != (m, c)
                                         or residual.stride(1) != 1):
                raise ValueError("residual must be a BF16 tensor [M, %d] with a contiguous last dimension" % c)
            d.bias_bf16 = bias.data_ptr() if bias is not None else None
            d.residual_bf16 = residual.data_ptr() if residual is not None else None
            d.ldr = (residual.stride(0) if m > 1 else c) if residual is not None else 0
            d.y_bf16, d.ldy = y.data_ptr(), (y.stride(0) if m > 1 else c)
            self._keep.append((x, q, s, bias, residual, y))
            self.ys.append(y)
        self.device = items[0]["x"].device if items else None
        self.chained = chained
        if chained:
            self._opts = ChainOpts(int(wait_us), int(phantom_workgroups), int(mode))
            self.workspace = None
            self.chain_ws = None
            if self.count:
                nbytes = int(load().mxfp4_woq_gemm_chain_workspace_bytes())
                self.chain_ws = torch.empty((nbytes,), dtype=torch.uint8, device=self.device)
                self.chain_reset()
            return
        need = int(load().mxfp4_woq_gemm_grouped_workspace_bytes(self._descs, self.count))
        self.workspace = torch.empty((need,), dtype=torch.uint8, device=self.device) if need else None

    def chain_reset(self) -> None:
        """Prepare the chain workspace again (after a wait that was given up)."""
        with _on(self.device):
            _check(load().mxfp4_woq_gemm_chain_init(_ptr(self.chain_ws), self.chain_ws.numel(), _stream()))

    def chain_status(self) -> int:
        """The chain workspace's status word (0: every wait so far was met); synchronises."""
        return int(self.chain_ws[CHAIN_STATUS_OFFSET:CHAIN_STATUS_OFFSET + 4].view(torch.int32).item())

    def run(self) -> None:
        if self.count == 0:
            return
        if self.chained:
            with _on(self.device):
                _check(load().mxfp4_woq_gemm_chain(self._descs, self.count, _ptr(self.chain_ws),
                                                   self.chain_ws.numel(), ctypes.byref(self._opts), _stream()))
            return
        with _on(self.device):
            _check(load().mxfp4_woq_gemm_grouped(
                self._descs, self.count, _ptr(self.workspace),
                self.workspace.numel() if self.workspace is not None else 0, _stream()))


class TiledWeights:
    """The tile-major copy of an MXFP4 weight pair (``mxfp4_tile_repack``) with its logical shape."""

    def __init__(self, q_tiled: torch.Tensor, s_tiled: torch.Tensor, n: int, k: int):
        self.q, self.s, self.n, self.k = q_tiled, s_tiled, n, k


def mxfp4_tile_repack(q: torch.Tensor, s: torch.Tensor) -> TiledWeights:
    _dev(q)
    if q.dtype != torch.uint8 or s.dtype != torch.uint8 or not q.is_contiguous() or not s.is_contiguous():
        raise ValueError("q and s must be contiguous uint8 tensors")
    n, k = q.shape[0], q.shape[1] * 2
    qt = torch.empty((int(load().mxfp4_tile_repack_q_bytes(n, k)),), dtype=torch.uint8, device=q.device)
    st = torch.empty((int(load().mxfp4_tile_repack_s_bytes(n, k)),), dtype=torch.uint8, device=q.device)
    with _on(q.device):
        _check(load().mxfp4_tile_repack(_ptr(q), _ptr(s), n, k, _ptr(qt), _ptr(st), _stream()))
    return TiledWeights(qt, st, n, k)


def _tiled_shapes(x: torch.Tensor, w: TiledWeights):
    _dev(x)
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1 or x.shape[1] != w.k:
        raise ValueError("x must be a 2-D BF16 tensor [M, %d] with a contiguous last dimension" % w.k)
    m = x.shape[0]
    return m, w.n, w.k, (x.stride(0) if m > 1 else w.k)


def mxfp4_woq_gemm_tiled(x: torch.Tensor, w: TiledWeights, y: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The product on the tile-major copy; with ``workspace`` (uint8, ``mxfp4_woq_gemm_workspace_bytes``)
    through ``mxfp4_woq_gemm_tiled_ws``, which also takes the shapes that need K split."""
    if y is None:
        y = _product(_TILED, x, w.q, w.s, w.n, w.k, False, None, 0, None, 0, workspace)
        if y is not None:
            return y
    m, n, k, ldx = _tiled_shapes(x, w)
    if y is None:
        y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    ldy = y.stride(0) if m > 1 else n
    with _on(x.device):
        if workspace is None:
            _check(load().mxfp4_woq_gemm_tiled(_ptr(x), m, ldx, _ptr(w.q), _ptr(w.s), n, k, _ptr(y), ldy, _stream()))
        else:
            _check(load().mxfp4_woq_gemm_tiled_ws(_ptr(x), m, ldx, _ptr(w.q), _ptr(w.s), n, k, _ptr(y), ldy,
                                                 _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                 _stream()))
    return y


def mxfp4_woq_gemm_tiled_fused(x: torch.Tensor, w: TiledWeights, bias: Optional[torch.Tensor] = None,
                               act: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
                               y: Optional[torch.Tensor] = None) -> torch.Tensor:
    if y is None:
        y = _product(_TILED, x, w.q, w.s, w.n, w.k, True, bias, act, residual, 0, None)
        if y is not None:
            return y
    m, n, k, ldx = _tiled_shapes(x, w)
    c = n // 2 if act == ACT_SWIGLU else n
    if bias is not None and (bias.dtype != torch.bfloat16 or bias.dim() != 1 or bias.shape[0] != n
                             or not bias.is_contiguous() or bias.device != x.device):
        raise ValueError("bias must be a contiguous BF16 tensor [N] on the device of x")
    if residual is not None and (residual.dtype != torch.bfloat16 or residual.dim() != 2
                                 or residual.shape != (m, c) or residual.stride(1) != 1
                                 or residual.device != x.device):
        raise ValueError("residual must be a BF16 tensor [M, %d] with a contiguous last dimension" % c)
    if y is None:
        y = torch.empty((m, c), dtype=torch.bfloat16, device=x.device)
    ldy = y.stride(0) if m > 1 else c
    ldr = (residual.stride(0) if m > 1 else c) if residual is not None else 0
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_tiled_fused(_ptr(x), m, ldx, _ptr(w.q), _ptr(w.s), n, k, _ptr(bias), act,
                                                _ptr(residual), ldr, _ptr(y), ldy, _stream()))
    return y


def mxfp4_woq_gemm_tiled_argmax(x: torch.Tensor, w: TiledWeights, workspace: Optional[torch.Tensor] = None,
                                out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                                ) -> Tuple[torch.Tensor, torch.Tensor]:
    m, n, k, ldx = _tiled_shapes(x, w)
    if workspace is None:
        workspace = torch.empty((mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k),), dtype=torch.uint8,
                                device=x.device)
    if out is None:
        idx = torch.empty((m,), dtype=torch.int32, device=x.device)
        val = torch.empty((m,), dtype=torch.float32, device=x.device)
    else:
        idx, val = out
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_tiled_argmax(_ptr(x), m, ldx, _ptr(w.q), _ptr(w.s), n, k, _ptr(idx),
                                                 _ptr(val), _ptr(workspace),
                                                 workspace.numel() * workspace.element_size(), _stream()))
    return idx, val


def mxfp4_woq_gemm_tiled_verify(x: torch.Tensor, w: TiledWeights, draft: Optional[torch.Tensor],
                                workspace: Optional[torch.Tensor] = None):
    got = _verify(_TILED, x, w.q, w.s, w.n, w.k, draft, workspace)
    if got is not None:
        return got
    m, n, k, ldx = _tiled_shapes(x, w)
    workspace, accept, idx, val = _verify_buffers(x, m, draft, mxfp4_woq_gemm_argmax_workspace_bytes(m, n, k),
                                                  workspace)
    with _on(x.device):
        _check(load().mxfp4_woq_gemm_tiled_verify(_ptr(x), m, ldx, _ptr(w.q), _ptr(w.s), n, k, _ptr(draft),
                                                 _ptr(accept), _ptr(idx), _ptr(val), _ptr(workspace),
                                                 workspace.numel() * workspace.element_size(), _stream()))
    return accept, idx, val


def mxfp4_bf16_gemm_verify(x: torch.Tensor, w: torch.Tensor, draft: Optional[torch.Tensor],
                           workspace: Optional[torch.Tensor] = None):
    """The same with unquantised BF16 weights."""
    got = _verify(_BF16, x, w, None, 0, 0, draft, workspace)
    if got is not None:
        return got
    m, n, k, ldx, ldw = _bf16_shapes(x, w)
    workspace, accept, idx, val = _verify_buffers(x, m, draft, mxfp4_bf16_gemm_argmax_workspace_bytes(m, n, k),
                                                  workspace)
    with _on(x.device):
        _check(load().mxfp4_bf16_gemm_verify(_ptr(x), m, ldx, _ptr(w), n, k, ldw, _ptr(draft), _ptr(accept),
                                            _ptr(idx), _ptr(val), _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream()))
    return accept, idx, val


def mxfp4_diag_stream_read(src: torch.Tensor, sink: torch.Tensor) -> None:
    with _on(src.device):
        _check(load().mxfp4_diag_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream()))


def mxfp4_diag_stream_copy(src: torch.Tensor, dst: torch.Tensor) -> None:
    with _on(src.device):
        _check(load().mxfp4_diag_stream_copy(_ptr(src), _ptr(dst), src.numel() * src.element_size(), _stream()))


# ---- the paged cache ------------------------------------------------------------------------------------------------


class KvCache(NamedTuple):
    """Keys and values in MXFP4: ``kq``, ``vq`` uint8 ``[pages, heads, page, dim/2]``, ``ks``, ``vs`` uint8
    ``[pages, heads, page, dim/32]``; pages may lie further apart (``x[:, layer]`` of an array with all layers)."""
    kq: torch.Tensor
    ks: torch.Tensor
    vq: torch.Tensor
    vs: torch.Tensor


class KvPool(NamedTuple):
    """Who holds which page: ``refs`` int32 ``[pages]``, ``free`` int32 ``[ceil(pages / 32)]``, a bit per free page."""
    refs: torch.Tensor
    free: torch.Tensor


def mxfp4_kv_cache(pages: int, heads: int, page: int, dim: int, layers: Optional[int] = None, device="cuda") -> KvCache:
    """A cache of zeros.  With ``layers`` the arrays are ``[pages, layers, heads, page, ...]``; ``mxfp4_kv_layer`` gives a
    layer's cache, ``mxfp4_kv_all_layers`` the one whose pages hold every layer (for extend, compact and copies)."""
    mid = (heads,) if layers is None else (layers, heads)
    return KvCache(*(torch.zeros((pages, *mid, page, dim // n), dtype=torch.uint8, device=device) for n in (2, 32, 2, 32)))


def mxfp4_kv_layer(cache: KvCache, layer: int) -> KvCache:
    return KvCache(*(x[:, layer] for x in cache))


def mxfp4_kv_all_layers(cache: KvCache) -> KvCache:
    """The same memory with layers and heads in one dimension.  Some of the heads alone cannot be seen so (a copy would take what
    extend, compact and copies store and lose it)."""
    for x in cache:
        if x.dim() != 5 or (x.shape[1] > 1 and x.shape[2] > 0 and x.stride(1) != x.shape[2] * x.stride(2)):
            raise ValueError("a cache with layers is [pages, layers, heads, page, ...] with all heads of a layer in a row: got %r with strides %r" % (
                tuple(x.shape), x.stride()))
    return KvCache(*(x.flatten(1, 2) for x in cache))


def mxfp4_kv_pool(pages: int, device="cuda") -> KvPool:
    """A pool whose pages are all free."""
    words = [-1] * (pages // 32) + ([(1 << pages % 32) - 1] if pages % 32 else [])
    return KvPool(torch.zeros((pages,), dtype=torch.int32, device=device),
                  torch.tensor(words, dtype=torch.int64).to(torch.int32).to(device))


def _kv_cache_desc(c: KvCache) -> KvCacheDesc:
    _dev(c.kq)
    if c.kq.dim() != 4 or c.ks.dim() != 4:
        raise ValueError("the cache's arrays are [pages, heads, page, dim/2] and [pages, heads, page, dim/32]")
    pages, heads, page, half = c.kq.shape
    for x, want, like in ((c.kq, half, c.kq), (c.ks, half // 16, c.ks), (c.vq, half, c.kq), (c.vs, half // 16, c.ks)):
        if (x.dtype != torch.uint8 or tuple(x.shape) != (pages, heads, page, want) or x.device != c.kq.device
                or x.stride()[1:] != (page * want, want, 1) or x.stride(0) != like.stride(0)):
            raise ValueError("the cache's arrays must be uint8, of one number of pages, heads and tokens, on one device, and contiguous "
                             "within a page: got %r" % [(tuple(x.shape), x.stride(), x.dtype) for x in c])
    return KvCacheDesc(c.kq.data_ptr(), c.ks.data_ptr(), c.vq.data_ptr(), c.vs.data_ptr(), pages,
                       c.kq.stride(0) if pages > 1 else heads * page * half, c.ks.stride(0) if pages > 1 else heads * page * (half // 16),
                       heads, page, half * 2, 0)


def _kv_ints(t: Optional[torch.Tensor], device, what: str, *shape) -> None:
    if t is not None and (t.dtype != torch.int32 or t.device != device or t.dim() != len(shape) or not t.is_contiguous()
                          or any(n is not None and m != n for m, n in zip(t.shape, shape))):
        raise ValueError("%s must be a contiguous int32 tensor of shape %r on %s" % (what, shape, device))


def _kv_table(table: torch.Tensor, device) -> int:
    """The checks of a table; its row stride."""
    if table.dtype != torch.int32 or table.device != device or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be an int32 tensor [rows, width] on %s with contiguous rows" % (device,))
    return table.stride(0) if table.shape[0] > 1 else table.shape[1]


def _kv_rows_desc(table, lens, starts, tokens: int, device) -> KvRowsDesc:
    ldt = _kv_table(table, device)
    rows = table.shape[0]
    _kv_ints(lens, device, "lens", rows)
    _kv_ints(starts, device, "starts", rows + 1)
    return KvRowsDesc(table.data_ptr(), ldt, table.shape[1], lens.data_ptr(), _ptr(starts), rows, tokens)


def _kv_tensor_desc(t: torch.Tensor, what: str, device, tokens: int, heads: Optional[int], dim: int) -> KvTensorDesc:
    if (t.dtype != torch.bfloat16 or t.device != device or t.dim() != 3 or t.shape[0] != tokens or t.shape[2] != dim
            or (heads is not None and t.shape[1] != heads) or t.stride(2) != 1):
        raise ValueError("%s must be a BF16 tensor [%d, %s, %d] on %s with a contiguous last dimension: got %r" % (
            what, tokens, "heads" if heads is None else heads, dim, device, tuple(t.shape)))
    return KvTensorDesc(t.data_ptr(), t.stride(0) if tokens > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0)


def mxfp4_kv_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
                    starts: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                    rope: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, positions: Optional[torch.Tensor] = None,
                    q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Stores the new tokens ``k``, ``v`` BF16 ``[tokens, heads, dim]`` of the sequences of ``table`` int32 ``[rows, width]`` at the
    ends of their lengths ``lens`` int32 ``[rows]`` (which count them already).  ``rope``: (cos, sin) float32 ``[length, d/2]``
    turns the first d elements of ``k``, and of ``q`` into the tensor that is returned, at the tokens' places or at
    ``positions`` int32 ``[tokens]``.  ``starts`` int32 ``[rows + 1]``: whose rows are whose; None: the same number each."""
    if q_out is None:
        got = (_kv or _kv_host()).append(cache, k, v, table, lens, starts, q, rope, positions)
        if got is not None:
            return got if q is not None else None
    c = _kv_cache_desc(cache)
    dev, tokens = cache.kq.device, k.shape[0]
    b = _kv_rows_desc(table, lens, starts, tokens, dev)
    kd, vd = _kv_tensor_desc(k, "k", dev, tokens, c.heads, c.dim), _kv_tensor_desc(v, "v", dev, tokens, c.heads, c.dim)
    qd = od = rd = None
    if q is not None:
        qd = _kv_tensor_desc(q, "q", dev, tokens, None, c.dim)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        od = _kv_tensor_desc(q_out, "q_out", dev, tokens, q.shape[1], c.dim)
    if rope is not None:
        cos, sin = rope
        if (cos.dim() != 2 or cos.shape != sin.shape or any(x.dtype != torch.float32 or x.device != dev or not x.is_contiguous() for x in rope)):
            raise ValueError("rope must be two contiguous float32 tensors [length, d/2] on %s" % (dev,))
        _kv_ints(positions, dev, "positions", tokens)
        rd = KvRopeDesc(cos.data_ptr(), sin.data_ptr(), _ptr(positions), cos.shape[0], 2 * cos.shape[1])
    elif positions is not None:
        raise ValueError("positions without rope")
    with _on(dev):
        _check(load().mxfp4_kv_append(c, b, kd, vd, qd, od, 0 if q is None else q.shape[1], rd, _stream()))
    return q_out if q is not None else None


def mxfp4_kv_read(cache: KvCache, table: torch.Tensor, lens: torch.Tensor, tokens: int, starts: Optional[torch.Tensor] = None,
                  out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The last tokens of the sequences, ``tokens`` in all, as the values that the cache holds: (k, v) BF16 ``[tokens, heads, dim]``."""
    if out is None:
        out = (_kv or _kv_host()).read(cache, table, lens, tokens, starts)
        if out is not None:
            return out
    c = _kv_cache_desc(cache)
    dev = cache.kq.device
    b = _kv_rows_desc(table, lens, starts, tokens, dev)
    k, v = out if out is not None else (torch.empty((tokens, c.heads, c.dim), dtype=torch.bfloat16, device=dev) for _ in range(2))
    kd, vd = _kv_tensor_desc(k, "k", dev, tokens, c.heads, c.dim), _kv_tensor_desc(v, "v", dev, tokens, c.heads, c.dim)
    with _on(dev):
        _check(load().mxfp4_kv_read(c, b, kd, vd, _stream()))
    return k, v


# One workspace for each stream that attention has run on, as a program would keep it: its counters zeroed when it is made, left at
# zero by every call, and used by calls that the stream runs one after the other.  Under graph capture a call gets one of
# its own, which belongs to the graph.
_kv_workspaces = {}


def _kv_workspace(device: torch.device, stream: int, need: int) -> torch.Tensor:
    key = stream * 64 + device.index
    capturing = torch.cuda.is_current_stream_capturing()
    ws = None if capturing else _kv_workspaces.get(key)
    if ws is None or ws.numel() < need:
        ws = torch.empty((need,), dtype=torch.uint8, device=device)
        ws[:4 * KV_COUNTERS].zero_()
        if not capturing:
            _kv_workspaces[key] = ws
    return ws


def mxfp4_kv_attention_workspace_bytes(cache: KvCache, rows: int, tokens: int, q_heads: int) -> int:
    """Bytes of a workspace for this many sequences and new tokens (its first ``4 * KV_COUNTERS`` bytes must be zero before the first call)."""
    return int(load().mxfp4_kv_attention_workspace_bytes(_kv_cache_desc(cache), KvRowsDesc(None, 0, 0, None, None, rows, tokens), q_heads))


def mxfp4_kv_attention(q: torch.Tensor, cache: KvCache, table: torch.Tensor, lens: torch.Tensor,
                       starts: Optional[torch.Tensor] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                       tree: Optional[torch.Tensor] = None, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None):
    """Attention of the new tokens ``q`` BF16 ``[tokens, q_heads, dim]`` over the cached ones (the new ones among them, see
    ``mxfp4_kv_append``); ``scale``: dim ** -0.5.  ``window`` > 0: only the last ``window`` tokens.  ``tree`` int64 ``[tokens]``: bit m says
    that the query sees new token m of its sequence, in place of the causal rule.  Returns BF16 ``[tokens, q_heads, dim]``, with
    ``return_lse`` also the logarithms of the softmax sums, float32 ``[tokens, q_heads]``.  ``workspace``: None takes the one that the binding
    keeps for the current stream."""
    if out is None and workspace is None:
        got = (_kv or _kv_host()).attention(q, cache, table, lens, starts, scale, causal, window, tree, return_lse, _kv_workspaces)
        if got is not None:
            return got
    c = _kv_cache_desc(cache)
    dev = cache.kq.device
    tokens = q.shape[0]
    b = _kv_rows_desc(table, lens, starts, tokens, dev)
    qd = _kv_tensor_desc(q, "q", dev, tokens, None, c.dim)
    q_heads = q.shape[1]
    if out is None:
        out = torch.empty((tokens, q_heads, c.dim), dtype=torch.bfloat16, device=dev)
    od = _kv_tensor_desc(out, "out", dev, tokens, q_heads, c.dim)
    if tree is not None and (tree.dtype != torch.int64 or tree.device != dev or tuple(tree.shape) != (tokens,) or not tree.is_contiguous()):
        raise ValueError("tree must be a contiguous int64 tensor [%d] on %s" % (tokens, dev))
    lse = torch.empty((tokens, q_heads), dtype=torch.float32, device=dev) if return_lse else None
    args = KvAttentionArgs(qd, od, _ptr(lse), _ptr(tree), q_heads, window, c.dim ** -0.5 if scale is None else scale, int(causal))
    with _on(dev):
        lib, stream = load(), _stream()
        if workspace is None:
            workspace = _kv_workspace(dev, stream, int(lib.mxfp4_kv_attention_workspace_bytes(c, b, q_heads)))
        _check(lib.mxfp4_kv_attention(c, b, args, workspace.data_ptr(), workspace.numel() * workspace.element_size(), stream))
    return (out, lse) if return_lse else out


def _kv_pool_desc(pool: KvPool, cache: KvCache, table: torch.Tensor, lens: torch.Tensor) -> KvPoolDesc:
    _dev(pool.refs)
    dev, pages = pool.refs.device, pool.refs.shape[0]
    _kv_ints(pool.refs, dev, "refs", None)
    _kv_ints(pool.free, dev, "free", (pages + 31) // 32)
    ldt = _kv_table(table, dev)
    _kv_ints(lens, dev, "lens", table.shape[0])
    return KvPoolDesc(pool.refs.data_ptr(), pool.free.data_ptr(), pages, cache.kq.shape[2], table.data_ptr(), ldt, table.shape[1],
                      table.shape[0], lens.data_ptr())


def _kv_two_lists(a: torch.Tensor, b: torch.Tensor, names: str, device) -> int:
    _kv_ints(a, device, names, None)
    _kv_ints(b, device, names, a.shape[0])
    return a.shape[0]


def mxfp4_kv_fork(pool: KvPool, cache: KvCache, table: torch.Tensor, lens: torch.Tensor, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Sequence ``dst[i]`` (empty) becomes a second owner of what sequence ``src[i]`` holds; nothing is copied."""
    if (_kv or _kv_host()).pages(0, *pool, cache, table, lens, src, dst):
        return
    p, n = _kv_pool_desc(pool, cache, table, lens), _kv_two_lists(src, dst, "src and dst", pool.refs.device)
    with _on(pool.refs.device):
        _check(load().mxfp4_kv_fork(p, _ptr(src), _ptr(dst), n, _stream()))


def mxfp4_kv_extend(pool: KvPool, cache: KvCache, table: torch.Tensor, lens: torch.Tensor, rows: torch.Tensor, add: torch.Tensor
                    ) -> torch.Tensor:
    """Room for ``add[i]`` more tokens of sequence ``rows[i]``: pages are taken, a shared last page becomes a copy, ``lens`` grows.
    ``cache``: its pages hold all that belongs to a token (all layers).  Returns int32 ``[1]`` on the device: 0, or what is missing
    (pages, or -1 for a table that is too narrow); then nothing has changed."""
    got = (_kv or _kv_host()).pages(2, *pool, cache, table, lens, rows, add)
    if got is not None:
        return got
    dev = pool.refs.device
    if cache.kq.device != dev:                                        # its pages are copied by a kernel of the pool's device
        raise ValueError("the cache must be on the pool's device %s, it is on %s" % (dev, cache.kq.device))
    p, n = _kv_pool_desc(pool, cache, table, lens), _kv_two_lists(rows, add, "rows and add", dev)
    got = torch.empty((2 * n + 1,), dtype=torch.int32, device=dev)
    with _on(dev):
        _check(load().mxfp4_kv_extend(p, _kv_cache_desc(cache), _ptr(rows), _ptr(add), n, got.data_ptr() + 4, got.data_ptr(), _stream()))
    return got[:1]


def mxfp4_kv_release(pool: KvPool, cache: KvCache, table: torch.Tensor, lens: torch.Tensor, rows: torch.Tensor, keep: torch.Tensor) -> None:
    """Sequence ``rows[i]`` is cut down to its first ``keep[i]`` tokens (0: all of it is given up); pages that nobody holds any more are free."""
    if (_kv or _kv_host()).pages(1, *pool, cache, table, lens, rows, keep):
        return
    p, n = _kv_pool_desc(pool, cache, table, lens), _kv_two_lists(rows, keep, "rows and keep", pool.refs.device)
    with _on(pool.refs.device):
        _check(load().mxfp4_kv_release(p, _ptr(rows), _ptr(keep), n, _stream()))


def mxfp4_kv_compact(cache: KvCache, table: torch.Tensor, base: torch.Tensor, keep: torch.Tensor, counts: torch.Tensor) -> None:
    """Token ``base[b] + keep[b, i]`` of sequence b moves to ``base[b] + i`` for i below ``counts[b]``; ``keep`` ascends."""
    if (_kv or _kv_host()).compact(cache, table, base, keep, counts):
        return
    c, dev = _kv_cache_desc(cache), cache.kq.device
    ldt, rows = _kv_table(table, dev), table.shape[0]
    _kv_ints(base, dev, "base", rows)
    _kv_ints(counts, dev, "counts", rows)
    _kv_ints(keep, dev, "keep", rows, None)
    with _on(dev):
        _check(load().mxfp4_kv_compact(c, table.data_ptr(), ldt, table.shape[1], _ptr(base), _ptr(keep), keep.shape[1], _ptr(counts), rows,
                                       _stream()))


def mxfp4_kv_copy_pages(cache: KvCache, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Page ``src[i]`` is copied to page ``dst[i]``."""
    c, n = _kv_cache_desc(cache), _kv_two_lists(src, dst, "src and dst", cache.kq.device)
    with _on(cache.kq.device):
        _check(load().mxfp4_kv_copy_pages(c, _ptr(src), _ptr(dst), n, _stream()))
