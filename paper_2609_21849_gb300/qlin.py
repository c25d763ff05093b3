"""Thin ctypes binding of libqlin (include/qlin.h): same names, argument
marshalling only.  Every step runs in the library's CUDA kernels; PyTorch
supplies device memory and the current stream.  There is no CPU fallback: if
the library is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
import types
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libqlin.so")

QLIN_FMT_NVFP4 = 1
QLIN_FMT_FP8 = 2
QLIN_BF16, QLIN_FP16 = 1, 2
QLIN_ACT_NONE, QLIN_ACT_RELU, QLIN_ACT_SILU, QLIN_ACT_GELU_TANH, QLIN_ACT_GELU = range(5)
QLIN_ROPE_INTERLEAVED, QLIN_ROPE_HALF = 0, 1
QLIN_ROPE_NONE, QLIN_ROPE_LINEAR, QLIN_ROPE_NTK, QLIN_ROPE_YARN = range(4)
QLIN_CACHE_BF16, QLIN_CACHE_FP16, QLIN_CACHE_E4M3 = 1, 2, 3
STATUS = {0: "QLIN_OK", 1: "QLIN_ERR_INVALID_ARG", 2: "QLIN_ERR_UNSUPPORTED",
          3: "QLIN_ERR_MISALIGNED", 4: "QLIN_ERR_CUDA", 5: "QLIN_ERR_TIMEOUT",
          6: "QLIN_ERR_WORKSPACE"}

# Every function declared in include/qlin.h.
EXPORTS = ("qlin_nvfp4_scale_bytes", "qlin_workspace_size", "qlin_quantize_act_nvfp4",
           "qlin_quantize_act_fp8", "qlin_quantize_weight", "qlin_gemm_nvfp4", "qlin_gemm_fp8",
           "qlin_linear_fused", "qlin_linear_fused_fp8", "qlin_linear_dynamic", "qlin_gemm_bf16",
           "qlin_gemm_fp16", "qlin_quantize_act_nvfp4_noalloc",
           "qlin_rmsnorm", "qlin_rmsnorm_fp8", "qlin_rmsnorm_nvfp4",
           "qlin_linear_nvfp4", "qlin_linear_fp8", "qlin_linear_bf16", "qlin_linear_fp16",
           "qlin_rope", "qlin_rope_turns",
           "qlin_fp8_block_scales", "qlin_quantize_fp8_block", "qlin_linear_fp8_block",
           "qlin_cache_append", "qlin_cache_attention", "qlin_cache_attention_workspace_size",
           "qlin_sync_status", "qlin_selftest_bounded_wait",
           "qlin_set_wait_timeout_ns", "qlin_status_str", "qlin_last_error")


class QlinError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}" + (f" ({detail})" if detail else ""))


class NVFP4Desc(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("tensor_scale", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("K", ctypes.c_int64)]


class FP8Desc(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("K", ctypes.c_int64),
                ("per_channel", ctypes.c_int32)]


class RMSNormDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "residual", "sum", "weight")]
                + [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "sum_stride", "M", "K")]
                + [("eps", ctypes.c_float), ("dtype", ctypes.c_int32)])


class EpilogueDesc(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("residual_stride", ctypes.c_int64), ("act", ctypes.c_int32)]


class RopeDesc(ctypes.Structure):
    _fields_ = ([("x", ctypes.c_void_p), ("y", ctypes.c_void_p)]
                + [(n, ctypes.c_int64) for n in ("x_token_stride", "x_head_stride", "y_token_stride",
                                                 "y_head_stride", "tokens", "heads")]
                + [("positions", ctypes.c_void_p), ("position_token_stride", ctypes.c_int64),
                   ("position_axis_stride", ctypes.c_int64), ("turns", ctypes.c_void_p),
                   ("magnitude", ctypes.c_float)]
                + [(n, ctypes.c_int32) for n in ("head_dim", "rot_dim", "position_bits", "axes")]
                + [("axis_pairs", ctypes.c_int32 * 4)]
                + [(n, ctypes.c_int32) for n in ("layout", "inverse", "dtype")])


class FP8BlockDesc(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("K", ctypes.c_int64), ("block_rows", ctypes.c_int32)]


class CacheDesc(ctypes.Structure):
    _fields_ = ([("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]
                + [(n, ctypes.c_int64) for n in ("k_page_stride", "k_slot_stride", "k_head_stride", "v_page_stride",
                                                 "v_slot_stride", "v_head_stride")]
                + [("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("cached", "q_start", "k_scale", "v_scale")]
                + [(n, ctypes.c_int32) for n in ("sequences", "pages", "page_size", "table_width", "heads",
                                                 "head_dim", "format")])


class CacheAppendDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "q", "q_out")]
                + [(n, ctypes.c_int64) for n in ("k_token_stride", "k_head_stride", "v_token_stride",
                                                 "v_head_stride", "q_token_stride", "q_head_stride",
                                                 "q_out_token_stride", "q_out_head_stride", "tokens")]
                + [("positions", ctypes.c_void_p), ("position_token_stride", ctypes.c_int64),
                   ("position_axis_stride", ctypes.c_int64), ("turns", ctypes.c_void_p),
                   ("magnitude", ctypes.c_float)]
                + [(n, ctypes.c_int32) for n in ("q_heads", "rot_dim", "position_bits", "axes")]
                + [("axis_pairs", ctypes.c_int32 * 4)] + [(n, ctypes.c_int32) for n in ("layout", "dtype")])


class CacheAttentionDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "out", "lse", "mask")]
                + [(n, ctypes.c_int64) for n in ("q_token_stride", "q_head_stride", "out_token_stride",
                                                 "out_head_stride", "mask_stride", "tokens")]
                + [("scale", ctypes.c_float)]
                + [(n, ctypes.c_int32) for n in ("q_heads", "mask_words", "dtype")])


# The descriptors as packed bytes, the form the calls below hand over: the
# struct's layout, built in a third of the time of a ctypes Structure and its
# reference (0.2 against 0.6 us; a call's host time is a few microseconds).
_pack_nvfp4 = struct.Struct("=QQQqq").pack
_pack_fp8 = struct.Struct("=QQqqi4x").pack
assert struct.calcsize("=QQQqq") == ctypes.sizeof(NVFP4Desc)
assert struct.calcsize("=QQqqi4x") == ctypes.sizeof(FP8Desc)
_pack_rmsnorm = struct.Struct("=QQQQqqqqqfi").pack
_pack_epilogue = struct.Struct("=QQqi4x").pack
_pack_rope = struct.Struct("=QQqqqqqqQqqQf11i").pack
_pack_fp8_block = struct.Struct("=QQqqi4x").pack
_pack_cache = struct.Struct("=QQ6qQqQQQQ7i4x").pack
_pack_append = struct.Struct("=QQQQ9qQqqQf10i4x").pack
_pack_attention = struct.Struct("=QQQQ6qf3i").pack
assert struct.calcsize("=QQqqi4x") == ctypes.sizeof(FP8BlockDesc)
assert struct.calcsize("=QQ6qQqQQQQ7i4x") == ctypes.sizeof(CacheDesc)
assert struct.calcsize("=QQQQ9qQqqQf10i4x") == ctypes.sizeof(CacheAppendDesc)
assert struct.calcsize("=QQQQ6qf3i") == ctypes.sizeof(CacheAttentionDesc)
assert struct.calcsize("=QQQQqqqqqfi") == ctypes.sizeof(RMSNormDesc)
assert struct.calcsize("=QQqi4x") == ctypes.sizeof(EpilogueDesc)
assert struct.calcsize("=QQqqqqqqQqqQf11i") == ctypes.sizeof(RopeDesc)

_lock = threading.Lock()
_lib = None


def _library():
    lib = _lib
    return lib if lib is not None else load_library()


def load_library(path: str = LIB_PATH):
    """Load libqlin.so (built by ``paper_2609_21849_gb300.build``)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(path):
            raise RuntimeError(f"libqlin is not built ({path} missing); run "
                               "python -m paper_2609_21849_gb300.build")
        lib = ctypes.CDLL(path)
        i64, p, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
        sig = {
            "qlin_nvfp4_scale_bytes": (sz, [i64, i64]),
            "qlin_workspace_size": (sz, [i64, i64]),
            "qlin_quantize_act_nvfp4": (ctypes.c_int, [p, i64, i64, p, ctypes.POINTER(NVFP4Desc), p, sz, p]),
            "qlin_quantize_act_fp8": (ctypes.c_int, [p, i64, i64, p, ctypes.POINTER(FP8Desc), p, sz, p]),
            "qlin_quantize_weight": (ctypes.c_int, [p, i64, i64, ctypes.c_int, p, p, sz, p]),
            "qlin_gemm_nvfp4": (ctypes.c_int, [ctypes.POINTER(NVFP4Desc), ctypes.POINTER(NVFP4Desc), p, p]),
            "qlin_gemm_fp8": (ctypes.c_int, [ctypes.POINTER(FP8Desc), ctypes.POINTER(FP8Desc), p, p]),
            "qlin_linear_fused": (ctypes.c_int, [ctypes.POINTER(NVFP4Desc), ctypes.POINTER(NVFP4Desc), p, p,
                                                 ctypes.POINTER(NVFP4Desc), i64, p]),
            "qlin_gemm_bf16": (ctypes.c_int, [p, i64, p, i64, i64, i64, p, p]),
            "qlin_gemm_fp16": (ctypes.c_int, [p, i64, p, i64, i64, i64, p, p]),
            "qlin_linear_fused_fp8": (ctypes.c_int, [ctypes.POINTER(FP8Desc), ctypes.POINTER(FP8Desc), p, p,
                                                     ctypes.POINTER(FP8Desc), i64, p]),
            "qlin_linear_dynamic": (ctypes.c_int, [ctypes.POINTER(NVFP4Desc), ctypes.POINTER(NVFP4Desc), p,
                                                   ctypes.POINTER(NVFP4Desc), p, sz, p]),
            "qlin_quantize_act_nvfp4_noalloc": (ctypes.c_int, [p, i64, i64, ctypes.POINTER(NVFP4Desc), p]),
            "qlin_rmsnorm": (ctypes.c_int, [ctypes.POINTER(RMSNormDesc), p, p]),
            "qlin_rmsnorm_fp8": (ctypes.c_int, [ctypes.POINTER(RMSNormDesc), p, ctypes.POINTER(FP8Desc), p]),
            "qlin_rmsnorm_nvfp4": (ctypes.c_int, [ctypes.POINTER(RMSNormDesc), p, ctypes.POINTER(NVFP4Desc), p]),
            "qlin_linear_nvfp4": (ctypes.c_int, [ctypes.POINTER(NVFP4Desc), ctypes.POINTER(NVFP4Desc),
                                                 ctypes.POINTER(EpilogueDesc), p, p,
                                                 ctypes.POINTER(NVFP4Desc), i64, p]),
            "qlin_linear_fp8": (ctypes.c_int, [ctypes.POINTER(FP8Desc), ctypes.POINTER(FP8Desc),
                                               ctypes.POINTER(EpilogueDesc), p, p,
                                               ctypes.POINTER(FP8Desc), i64, p]),
            "qlin_linear_bf16": (ctypes.c_int, [p, i64, p, i64, i64, i64, ctypes.POINTER(EpilogueDesc), p, p]),
            "qlin_linear_fp16": (ctypes.c_int, [p, i64, p, i64, i64, i64, ctypes.POINTER(EpilogueDesc), p, p]),
            "qlin_rope": (ctypes.c_int, [ctypes.POINTER(RopeDesc), p]),
            "qlin_rope_turns": (ctypes.c_int, [ctypes.c_int32, ctypes.c_double, ctypes.c_int32]
                                + [ctypes.c_double] * 4 + [p, ctypes.POINTER(ctypes.c_float)]),
            "qlin_fp8_block_scales": (sz, [i64, i64, ctypes.c_int32]),
            "qlin_quantize_fp8_block": (ctypes.c_int, [p, ctypes.c_int32, i64, ctypes.POINTER(FP8BlockDesc), p]),
            "qlin_linear_fp8_block": (ctypes.c_int, [ctypes.POINTER(FP8BlockDesc), ctypes.POINTER(FP8BlockDesc),
                                                     ctypes.POINTER(EpilogueDesc), p, p]),
            "qlin_cache_append": (ctypes.c_int, [ctypes.POINTER(CacheDesc), ctypes.POINTER(CacheAppendDesc), p]),
            "qlin_cache_attention": (ctypes.c_int, [ctypes.POINTER(CacheDesc), ctypes.POINTER(CacheAttentionDesc),
                                                    p, sz, p]),
            "qlin_cache_attention_workspace_size": (sz, []),
            "qlin_sync_status": (ctypes.c_int, [p]),
            "qlin_selftest_bounded_wait": (ctypes.c_int, [ctypes.c_uint64, p]),
            "qlin_set_wait_timeout_ns": (None, [ctypes.c_uint64]),
            "qlin_status_str": (ctypes.c_char_p, [ctypes.c_int]),
            "qlin_last_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        # the same functions with packed descriptors (bytes) for the calls
        d = ctypes.c_char_p
        packed = {
            "qlin_quantize_act_nvfp4": [p, i64, i64, p, d, p, sz, p],
            "qlin_quantize_act_fp8": [p, i64, i64, p, d, p, sz, p],
            "qlin_quantize_weight": [p, i64, i64, ctypes.c_int, d, p, sz, p],
            "qlin_gemm_nvfp4": [d, d, p, p],
            "qlin_gemm_fp8": [d, d, p, p],
            "qlin_linear_fused": [d, d, p, p, d, i64, p],
            "qlin_linear_fused_fp8": [d, d, p, p, d, i64, p],
            "qlin_linear_dynamic": [d, d, p, d, p, sz, p],
            "qlin_quantize_act_nvfp4_noalloc": [p, i64, i64, d, p],
            "qlin_rmsnorm": [d, p, p],
            "qlin_rmsnorm_fp8": [d, p, d, p],
            "qlin_rmsnorm_nvfp4": [d, p, d, p],
            "qlin_linear_nvfp4": [d, d, d, p, p, d, i64, p],
            "qlin_linear_fp8": [d, d, d, p, p, d, i64, p],
            "qlin_linear_bf16": [p, i64, p, i64, i64, i64, d, p, p],
            "qlin_linear_fp16": [p, i64, p, i64, i64, i64, d, p, p],
            "qlin_rope": [d, p],
            "qlin_quantize_fp8_block": [p, ctypes.c_int32, i64, d, p],
            "qlin_linear_fp8_block": [d, d, d, p, p],
            "qlin_cache_append": [d, d, p],
            "qlin_cache_attention": [d, d, p, sz, p],
        }
        lib.packed = types.SimpleNamespace()
        for name, args in packed.items():
            fn = lib[name]           # a function object of its own
            fn.restype = ctypes.c_int
            fn.argtypes = args
            setattr(lib.packed, name, fn)
        _lib = lib
        return lib


def _check(status: int, where: str):
    if status != 0:
        lib = _library()
        detail = lib.qlin_last_error().decode() if status == 4 else ""
        raise QlinError(status, where, detail)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # torch.cuda.current_stream() builds a Stream object (2.8 us); its raw
        # handle is all that a call needs
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _bf16_2d(x: torch.Tensor):
    if x.dtype != torch.bfloat16 or x.dim() != 2 or not x.is_contiguous() or not x.is_cuda:
        raise ValueError("expected a contiguous 2-D bf16 CUDA tensor")
    return x.shape[0], x.shape[1]


# ----------------------------------------------------------- containers ---

@dataclass
class NVFP4Tensor:
    """NVFP4 operand [rows, K] in device memory: packed e2m1 codes, E4M3 block
    scales in the tensor-core layout, fp32 tensor scale."""
    codes: torch.Tensor          # uint8 [rows, K/2]
    scales: torch.Tensor         # uint8 [qlin_nvfp4_scale_bytes(rows, K)]
    tensor_scale: torch.Tensor   # float32 [1]
    rows: int
    K: int

    def desc(self) -> NVFP4Desc:
        return NVFP4Desc(self.codes.data_ptr(), self.scales.data_ptr(),
                         self.tensor_scale.data_ptr(), self.rows, self.K)

    def packed(self) -> bytes:
        try:
            return _pack_nvfp4(self.codes.data_ptr(), self.scales.data_ptr(),
                               self.tensor_scale.data_ptr(), self.rows, self.K)
        except struct.error:   # no integer, or out of range: as the structure takes it
            return bytes(self.desc())


@dataclass
class FP8Tensor:
    """FP8 operand [rows, K]: E4M3 codes plus one fp32 scale (per_channel=0)
    or one per row (per_channel=1)."""
    codes: torch.Tensor          # uint8 [rows, K]
    scale: torch.Tensor          # float32 [1] or [rows]
    rows: int
    K: int
    per_channel: int

    def desc(self) -> FP8Desc:
        return FP8Desc(self.codes.data_ptr(), self.scale.data_ptr(), self.rows, self.K,
                       self.per_channel)

    def packed(self) -> bytes:
        try:
            return _pack_fp8(self.codes.data_ptr(), self.scale.data_ptr(), self.rows, self.K,
                             self.per_channel)
        except struct.error:
            return bytes(self.desc())


def qlin_nvfp4_scale_bytes(rows: int, K: int) -> int:
    return _library().qlin_nvfp4_scale_bytes(rows, K)


def qlin_workspace_size(M: int = 0, K: int = 0) -> int:
    return _library().qlin_workspace_size(M, K)


def alloc_nvfp4(rows: int, K: int, device="cuda") -> NVFP4Tensor:
    nb = qlin_nvfp4_scale_bytes(rows, K)
    if nb == 0:
        raise ValueError(f"invalid NVFP4 shape [{rows}, {K}]")
    return NVFP4Tensor(torch.empty((rows, K // 2), dtype=torch.uint8, device=device),
                       torch.zeros(nb, dtype=torch.uint8, device=device),
                       torch.zeros(1, dtype=torch.float32, device=device), rows, K)


def alloc_fp8(rows: int, K: int, per_channel: bool, device="cuda") -> FP8Tensor:
    return FP8Tensor(torch.empty((rows, K), dtype=torch.uint8, device=device),
                     torch.zeros(rows if per_channel else 1, dtype=torch.float32, device=device),
                     rows, K, 1 if per_channel else 0)


def alloc_workspace(device="cuda") -> torch.Tensor:
    return torch.zeros(qlin_workspace_size(), dtype=torch.uint8, device=device)


def _descriptor(t, desc) -> bytes:
    """The packed descriptor of an operand of another class than ours: its own
    desc(), which has to be of the right kind."""
    d = t.desc()
    if not isinstance(d, desc):
        raise ctypes.ArgumentError(f"expected {desc.__name__}, got {type(d).__name__}")
    return bytes(d)


def _nvfp4(t) -> bytes:
    return t.packed() if type(t) is NVFP4Tensor else _descriptor(t, NVFP4Desc)


def _fp8(t) -> bytes:
    return t.packed() if type(t) is FP8Tensor else _descriptor(t, FP8Desc)


# ------------------------------------------------------------ the calls ---

def qlin_quantize_act_nvfp4(x: torch.Tensor, static_scale: torch.Tensor | None = None,
                            out: NVFP4Tensor | None = None, workspace: torch.Tensor | None = None,
                            stream=None) -> NVFP4Tensor:
    M, K = _bf16_2d(x)
    out = out if out is not None else alloc_nvfp4(M, K, x.device)
    if static_scale is None and workspace is None:
        workspace = alloc_workspace(x.device)
    _check(_library().packed.qlin_quantize_act_nvfp4(
        x.data_ptr(), M, K, _ptr(static_scale), _nvfp4(out), _ptr(workspace),
        0 if workspace is None else workspace.numel(), _stream(stream)), "qlin_quantize_act_nvfp4")
    return out


def qlin_quantize_act_nvfp4_noalloc(x: torch.Tensor, out: NVFP4Tensor, stream=None) -> NVFP4Tensor:
    """Dynamic-scale NVFP4 quantization for callers that cannot allocate device
    memory: no workspace argument; the library keeps the amax scratch in its
    own static device array.  ``out`` must be supplied by the caller.  Calls
    that overlap on the GPU share that scratch and race; the first call on a
    device should come before any stream capture."""
    M, K = _bf16_2d(x)
    _check(_library().packed.qlin_quantize_act_nvfp4_noalloc(x.data_ptr(), M, K, _nvfp4(out),
                                                             _stream(stream)),
           "qlin_quantize_act_nvfp4_noalloc")
    return out


def qlin_quantize_act_fp8(x: torch.Tensor, static_scale: torch.Tensor | None = None,
                          out: FP8Tensor | None = None, workspace: torch.Tensor | None = None,
                          stream=None) -> FP8Tensor:
    M, K = _bf16_2d(x)
    out = out if out is not None else alloc_fp8(M, K, False, x.device)
    if static_scale is None and workspace is None:
        workspace = alloc_workspace(x.device)
    _check(_library().packed.qlin_quantize_act_fp8(
        x.data_ptr(), M, K, _ptr(static_scale), _fp8(out), _ptr(workspace),
        0 if workspace is None else workspace.numel(), _stream(stream)), "qlin_quantize_act_fp8")
    return out


def qlin_quantize_weight(w: torch.Tensor, fmt: int, out=None, workspace: torch.Tensor | None = None,
                         stream=None):
    N, K = _bf16_2d(w)
    if fmt == QLIN_FMT_NVFP4:
        out = out if out is not None else alloc_nvfp4(N, K, w.device)
        workspace = workspace if workspace is not None else alloc_workspace(w.device)
    elif fmt == QLIN_FMT_FP8:
        out = out if out is not None else alloc_fp8(N, K, True, w.device)
    else:
        raise ValueError("fmt must be QLIN_FMT_NVFP4 or QLIN_FMT_FP8")
    _check(_library().packed.qlin_quantize_weight(
        w.data_ptr(), N, K, fmt, bytes(out.desc()), _ptr(workspace),
        0 if workspace is None else workspace.numel(), _stream(stream)), "qlin_quantize_weight")
    return out


def _y_out(y, M, N, device):
    if y is None:
        return torch.empty((M, N), dtype=torch.bfloat16, device=device)
    if y.dtype != torch.bfloat16 or y.shape != (M, N) or not y.is_contiguous():
        raise ValueError("y must be a contiguous bf16 [M, N] tensor")
    return y


def qlin_gemm_nvfp4(A: NVFP4Tensor, W: NVFP4Tensor, y: torch.Tensor | None = None,
                    stream=None) -> torch.Tensor:
    y = _y_out(y, A.rows, W.rows, A.codes.device)
    _check(_library().packed.qlin_gemm_nvfp4(_nvfp4(A), _nvfp4(W), y.data_ptr(), _stream(stream)),
           "qlin_gemm_nvfp4")
    return y


def qlin_gemm_fp8(A: FP8Tensor, W: FP8Tensor, y: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
    y = _y_out(y, A.rows, W.rows, A.codes.device)
    _check(_library().packed.qlin_gemm_fp8(_fp8(A), _fp8(W), y.data_ptr(), _stream(stream)),
           "qlin_gemm_fp8")
    return y


def qlin_linear_fused(A: NVFP4Tensor, W: NVFP4Tensor, y: torch.Tensor | None,
                      next_scale: torch.Tensor | None, y_q: NVFP4Tensor | None,
                      rq_col0: int = 0, stream=None):
    _check(_library().packed.qlin_linear_fused(
        _nvfp4(A), _nvfp4(W), _ptr(y), _ptr(next_scale),
        _nvfp4(y_q) if y_q is not None else None, rq_col0, _stream(stream)),
        "qlin_linear_fused")
    return y, y_q


def qlin_linear_fused_fp8(A: FP8Tensor, W: FP8Tensor, y: torch.Tensor | None,
                          next_scale: torch.Tensor, y_q: FP8Tensor, rq_col0: int = 0, stream=None):
    """FP8 linear whose epilogue also writes the next layer's FP8 input
    (columns [rq_col0, rq_col0 + y_q.K) of bf16(y), static scale)."""
    _check(_library().packed.qlin_linear_fused_fp8(
        _fp8(A), _fp8(W), _ptr(y), _ptr(next_scale), _fp8(y_q), rq_col0, _stream(stream)),
        "qlin_linear_fused_fp8")
    return y, y_q


def _gemm16(name: str, dtype, a: torch.Tensor, w: torch.Tensor, y, stream):
    if a.dtype != dtype or w.dtype != dtype or a.dim() != 2 or a.stride(1) != 1:
        raise ValueError(f"a, w: {dtype} matrices with unit column stride")
    w = w.contiguous()
    M, K = a.shape
    N = w.shape[0]
    if y is None:
        y = torch.empty((M, N), dtype=dtype, device=a.device)
    elif y.dtype != dtype or not y.is_contiguous() or tuple(y.shape) != (M, N):
        raise ValueError(f"y: contiguous {dtype} [{M}, {N}]")
    _check(getattr(_library(), name)(_ptr(a), a.stride(0), _ptr(w), M, N, K, _ptr(y),
                                         _stream(stream)), name)
    return y


def qlin_gemm_bf16(a: torch.Tensor, w: torch.Tensor, y: torch.Tensor | None = None, stream=None):
    """y = a w^T for bf16 a [M, K] (rows may be strided: any view with unit
    column stride) and w [N, K]; bf16 y [M, N]."""
    return _gemm16("qlin_gemm_bf16", torch.bfloat16, a, w, y, stream)


def qlin_gemm_fp16(a: torch.Tensor, w: torch.Tensor, y: torch.Tensor | None = None, stream=None):
    """As qlin_gemm_bf16 with fp16 operands and an fp16 y."""
    return _gemm16("qlin_gemm_fp16", torch.float16, a, w, y, stream)


def qlin_linear_dynamic(A: NVFP4Tensor, W: NVFP4Tensor, y: torch.Tensor | None = None,
                        y_q: NVFP4Tensor | None = None, workspace: torch.Tensor | None = None,
                        stream=None):
    """y = A W^T (bf16) and y_q = NVFP4(y) with y's own dynamic tensor scale,
    the amax taken in the GEMM epilogue.  Returns (y, y_q)."""
    M, N = A.rows, W.rows
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=A.codes.device)
    if y_q is None:
        y_q = alloc_nvfp4(M, N, A.codes.device)
    if workspace is None:
        workspace = alloc_workspace(A.codes.device)
    _check(_library().packed.qlin_linear_dynamic(
        _nvfp4(A), _nvfp4(W), _ptr(y), _nvfp4(y_q), _ptr(workspace),
        workspace.numel(), _stream(stream)), "qlin_linear_dynamic")
    return y, y_q


# ------------------------------------- around the linears of a block ---

_FLOAT16 = {torch.bfloat16: QLIN_BF16, torch.float16: QLIN_FP16}


def _empty(shape, dtype, device, stream, make=torch.empty):
    """An output of a call on `stream`: allocated in that stream's order, so that
    memory that the current stream still uses is not handed out for it."""
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def _zero(t, stream):
    """Zeros in t, in the order of `stream`."""
    if stream is None:
        return t.zero_()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=t.device)
    with torch.cuda.stream(stream):
        return t.zero_()


# The checks below read each attribute of a tensor once and compare device indices, not
# device objects: a call's host time is a few microseconds.

def _rows16(t, name, dtype, M, K, dev):
    """The row stride of a 16-bit [M, K] matrix on device `dev` with adjacent columns."""
    if t.dtype is dtype and t.get_device() == dev:
        shape = t.shape
        if len(shape) == 2 and shape[0] == M and shape[1] == K:
            s0, s1 = t.stride()
            if s1 == 1 or K <= 1:
                return s0 if M > 1 else K
    raise ValueError(f"{name}: expected a {dtype} [{M}, {K}] tensor on cuda:{dev} with unit column stride")


def _vector16(t, name, dtype, n, dev):
    shape = t.shape
    if (t.dtype is not dtype or len(shape) != 1 or shape[0] != n or t.get_device() != dev
            or not t.is_contiguous()):
        raise ValueError(f"{name}: expected a contiguous {dtype} [{n}] tensor on cuda:{dev}")
    return t.data_ptr()


def _dense16(t, name, dtype, M, N, dev):
    shape = t.shape
    if (t.dtype is not dtype or len(shape) != 2 or shape[0] != M or shape[1] != N or t.get_device() != dev
            or not t.is_contiguous()):
        raise ValueError(f"{name}: expected a contiguous {dtype} [{M}, {N}] tensor on cuda:{dev}")
    return t.data_ptr()


def _scalar32(t, name, dev):
    """The address of a scale on device `dev` (an int is one already)."""
    if t is None or type(t) is int:
        return t
    p = t.data_ptr()
    if t.dtype is not torch.float32 or t.get_device() != dev or not p:
        raise ValueError(f"{name}: expected a float32 tensor on cuda:{dev}")
    return p


def _fp8_on(q, name, dev) -> bytes:
    """The packed descriptor of an FP8 operand, one of ours on device `dev`."""
    if type(q) is not FP8Tensor:
        return _descriptor(q, FP8Desc)
    codes, scale = q.codes, q.scale
    if codes.get_device() != dev or scale.get_device() != dev:
        raise ValueError(f"{name}: expected an operand on cuda:{dev}")
    try:
        return _pack_fp8(codes.data_ptr(), scale.data_ptr(), q.rows, q.K, q.per_channel)
    except struct.error:   # no integer, or out of range: as the structure takes it
        return bytes(q.desc())


def _nvfp4_on(q, name, dev) -> bytes:
    """The same of an NVFP4 operand."""
    if type(q) is not NVFP4Tensor:
        return _descriptor(q, NVFP4Desc)
    codes, scales, scale = q.codes, q.scales, q.tensor_scale
    if codes.get_device() != dev or scales.get_device() != dev or scale.get_device() != dev:
        raise ValueError(f"{name}: expected an operand on cuda:{dev}")
    try:
        return _pack_nvfp4(codes.data_ptr(), scales.data_ptr(), scale.data_ptr(), q.rows, q.K)
    except struct.error:
        return bytes(q.desc())


def _rmsnorm_args(x, weight, residual, eps, sum_out, stream):
    """(packed arguments, M, K, sum) of a norm call; sum is allocated where a
    residual comes without one."""
    dtype, dev, shape = x.dtype, x.get_device(), x.shape
    dt = _FLOAT16.get(dtype)
    if dt is None or len(shape) != 2 or dev < 0:
        raise ValueError("x: expected a 2-D bf16 or fp16 CUDA tensor")
    M, K = shape
    xs, rs, ss, rp, sp = _rows16(x, "x", dtype, M, K, dev), 0, 0, 0, 0
    if residual is not None:
        rs, rp = _rows16(residual, "residual", dtype, M, K, dev), residual.data_ptr()
        if sum_out is None:
            sum_out = _empty((M, K), dtype, x.device, stream)
        ss, sp = _rows16(sum_out, "sum_out", dtype, M, K, dev), sum_out.data_ptr()
    elif sum_out is not None:
        raise ValueError("sum_out without a residual")
    wp = 0 if weight is None else _vector16(weight, "weight", dtype, K, dev)
    return _pack_rmsnorm(x.data_ptr(), rp, sp, wp, xs, rs, ss, M, K, eps, dt), M, K, sum_out


def qlin_rmsnorm(x: torch.Tensor, weight: torch.Tensor | None = None,
                 residual: torch.Tensor | None = None, eps: float = 1e-6,
                 sum_out: torch.Tensor | None = None, y: torch.Tensor | None = None, stream=None):
    """(norm of x + residual in x's type, x + residual).  x, residual and sum_out are
    [M, K] with any row stride that is a multiple of 8; sum_out may be x or residual.
    Without a residual the second is None."""
    args, M, K, sum_out = _rmsnorm_args(x, weight, residual, eps, sum_out, stream)
    if y is None:
        y = _empty((M, K), x.dtype, x.device, stream)
    _check(_library().packed.qlin_rmsnorm(args, _dense16(y, "y", x.dtype, M, K, x.get_device()),
                                          _stream(stream)), "qlin_rmsnorm")
    return y, sum_out


def qlin_rmsnorm_fp8(x: torch.Tensor, weight: torch.Tensor | None = None,
                     residual: torch.Tensor | None = None, eps: float = 1e-6,
                     sum_out: torch.Tensor | None = None, static_scale: torch.Tensor | None = None,
                     out: FP8Tensor | None = None, stream=None):
    """The norm as an FP8 operand: one scale per row, found here, or the static
    tensor scale.  Returns (operand, x + residual) as qlin_rmsnorm does."""
    args, M, K, sum_out = _rmsnorm_args(x, weight, residual, eps, sum_out, stream)
    if out is None:
        rows = static_scale is None
        out = FP8Tensor(_empty((M, K), torch.uint8, x.device, stream),
                        _empty(M if rows else 1, torch.float32, x.device, stream), M, K, 1 if rows else 0)
    dev = x.get_device()
    _check(_library().packed.qlin_rmsnorm_fp8(args, _scalar32(static_scale, "static_scale", dev),
                                              _fp8_on(out, "out", dev), _stream(stream)),
           "qlin_rmsnorm_fp8")
    return out, sum_out


def qlin_rmsnorm_nvfp4(x: torch.Tensor, static_scale: torch.Tensor, weight: torch.Tensor | None = None,
                       residual: torch.Tensor | None = None, eps: float = 1e-6,
                       sum_out: torch.Tensor | None = None, out: NVFP4Tensor | None = None, stream=None):
    """The norm as an NVFP4 operand with the static tensor scale.  Returns
    (operand, x + residual) as qlin_rmsnorm does."""
    args, M, K, sum_out = _rmsnorm_args(x, weight, residual, eps, sum_out, stream)
    if out is None:
        nb = qlin_nvfp4_scale_bytes(M, K)
        if nb == 0:
            raise ValueError(f"invalid NVFP4 shape [{M}, {K}]")
        out = NVFP4Tensor(_empty((M, K // 2), torch.uint8, x.device, stream),
                          _empty(nb, torch.uint8, x.device, stream, torch.zeros),   # (padding too, as alloc_nvfp4)
                          _empty(1, torch.float32, x.device, stream), M, K)
    dev = x.get_device()
    _check(_library().packed.qlin_rmsnorm_nvfp4(args, _scalar32(static_scale, "static_scale", dev),
                                                _nvfp4_on(out, "out", dev), _stream(stream)),
           "qlin_rmsnorm_nvfp4")
    return out, sum_out


def _epilogue(bias, act, residual, dtype, M, N, dev):
    """The packed epilogue of a linear with an [M, N] output; None where it is empty."""
    if residual is None:
        if bias is None and act == QLIN_ACT_NONE:
            return None
        return _pack_epilogue(0 if bias is None else _vector16(bias, "bias", dtype, N, dev), 0, 0, act)
    return _pack_epilogue(0 if bias is None else _vector16(bias, "bias", dtype, N, dev), residual.data_ptr(),
                          _rows16(residual, "residual", dtype, M, N, dev), act)


def _linear_quantized(name, pack, A, W, bias, act, residual, y, next_scale, y_q, rq_col0, stream):
    M, N, codes = A.rows, W.rows, A.codes
    dev = codes.get_device()
    if dev < 0:
        raise ValueError("A: expected a CUDA operand")
    if (y_q is None) != (next_scale is None):
        raise ValueError("next_scale and y_q come together")
    if y is None and y_q is None:
        y = _empty((M, N), torch.bfloat16, codes.device, stream)
    yp = None if y is None else _dense16(y, "y", torch.bfloat16, M, N, dev)
    ep = _epilogue(bias, act, residual, torch.bfloat16, M, N, dev)
    _check(getattr(_library().packed, name)(
        pack(A, "A", dev), pack(W, "W", dev), ep, yp, _scalar32(next_scale, "next_scale", dev),
        None if y_q is None else pack(y_q, "y_q", dev), rq_col0, _stream(stream)), name)
    return y, y_q


def qlin_linear_nvfp4(A: NVFP4Tensor, W: NVFP4Tensor, bias: torch.Tensor | None = None,
                      act: int = QLIN_ACT_NONE, residual: torch.Tensor | None = None,
                      y: torch.Tensor | None = None, next_scale: torch.Tensor | None = None,
                      y_q: NVFP4Tensor | None = None, rq_col0: int = 0, stream=None):
    """y = act(A W^T + bias) + residual (bf16, one rounding) and, with next_scale and
    y_q, the next layer's NVFP4 input from columns [rq_col0, rq_col0 + y_q.K) of y.
    Returns (y, y_q); y None is allocated, or not written where y_q is given.
    residual may be y."""
    return _linear_quantized("qlin_linear_nvfp4", _nvfp4_on, A, W, bias, act, residual, y, next_scale, y_q,
                             rq_col0, stream)


def qlin_linear_fp8(A: FP8Tensor, W: FP8Tensor, bias: torch.Tensor | None = None,
                    act: int = QLIN_ACT_NONE, residual: torch.Tensor | None = None,
                    y: torch.Tensor | None = None, next_scale: torch.Tensor | None = None,
                    y_q: FP8Tensor | None = None, rq_col0: int = 0, stream=None):
    """As qlin_linear_nvfp4 with FP8 operands; A has one scale or one per row."""
    return _linear_quantized("qlin_linear_fp8", _fp8_on, A, W, bias, act, residual, y, next_scale, y_q,
                             rq_col0, stream)


def _linear16(name, dtype, a, w, bias, act, residual, y, stream):
    dev, shape = a.get_device(), a.shape
    if a.dtype is not dtype or len(shape) != 2 or dev < 0:
        raise ValueError(f"a: expected a 2-D {dtype} CUDA tensor")
    M, K = shape
    N = w.shape[0]
    wp = _dense16(w, "w", dtype, N, K, dev)
    lda = _rows16(a, "a", dtype, M, K, dev)
    if y is None:
        y = _empty((M, N), dtype, a.device, stream)
    _check(getattr(_library().packed, name)(a.data_ptr(), lda, wp, M, N, K,
                                            _epilogue(bias, act, residual, dtype, M, N, dev),
                                            _dense16(y, "y", dtype, M, N, dev), _stream(stream)), name)
    return y


def qlin_linear_bf16(a: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None,
                     act: int = QLIN_ACT_NONE, residual: torch.Tensor | None = None,
                     y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = act(a w^T + bias) + residual for bf16 a [M, K] (rows may be strided) and
    w [N, K], one rounding to bf16.  residual may be y."""
    return _linear16("qlin_linear_bf16", torch.bfloat16, a, w, bias, act, residual, y, stream)


def qlin_linear_fp16(a: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None,
                     act: int = QLIN_ACT_NONE, residual: torch.Tensor | None = None,
                     y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """As qlin_linear_bf16 in fp16."""
    return _linear16("qlin_linear_fp16", torch.float16, a, w, bias, act, residual, y, stream)


_LAYOUTS = {"interleaved": QLIN_ROPE_INTERLEAVED, "half": QLIN_ROPE_HALF}
_SCALINGS = {"none": QLIN_ROPE_NONE, "linear": QLIN_ROPE_LINEAR, "ntk": QLIN_ROPE_NTK, "yarn": QLIN_ROPE_YARN}


@dataclass
class RopePlan:
    """What the rotation needs beside positions: each pair's turns per position in
    units of 2^-64 turn, the layout ("interleaved" or "half"), the magnitude, and how
    many pairs follow each position axis."""
    turns: torch.Tensor          # int64 (the bits of uint64) [rot_dim / 2]
    layout: str
    magnitude: float
    axis_pairs: tuple

    @property
    def rot_dim(self) -> int:
        return 2 * self.turns.numel()


def qlin_rope_turns(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                    trained_length: float = 4096.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(turns as a host int64 tensor with uint64's bits, magnitude) of one axis."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling: one of {sorted(_SCALINGS)}")
    turns = torch.empty(max(rot_dim // 2, 0), dtype=torch.int64)
    mag = ctypes.c_float()
    _check(_library().qlin_rope_turns(rot_dim, base, _SCALINGS[scaling], factor, trained_length, beta_fast,
                                      beta_slow, turns.data_ptr(), ctypes.byref(mag)), "qlin_rope_turns")
    return turns, mag.value


def rope_plan(rot_dims, base: float = 10000.0, layout: str = "half", scaling: str = "none",
              factor: float = 1.0, trained_length: float = 4096.0, beta_fast: float = 32.0,
              beta_slow: float = 1.0, device="cuda") -> RopePlan:
    """A plan for heads whose first sum(rot_dims) elements turn; rot_dims is the
    rotated width, or one width per position axis (each with its own frequencies)."""
    if layout not in _LAYOUTS:
        raise ValueError(f"layout: one of {sorted(_LAYOUTS)}")
    dims = (rot_dims,) if isinstance(rot_dims, int) else tuple(rot_dims)
    if not 1 <= len(dims) <= 4:
        raise ValueError("one to four position axes")
    parts = [qlin_rope_turns(d, base, scaling, factor, trained_length, beta_fast, beta_slow) for d in dims]
    return RopePlan(torch.cat([t for t, _ in parts]).to(device), layout, parts[0][1],
                    tuple(d // 2 for d in dims))


def qlin_rope(x: torch.Tensor, positions: torch.Tensor, plan: RopePlan, out: torch.Tensor | None = None,
              inverse: bool = False, stream=None) -> torch.Tensor:
    """x [tokens, heads, head_dim] (any strides of tokens and heads, e.g. the q and k
    columns of a QKV output) with its rotary positions applied, or taken back
    (inverse: also the gradient).  positions: int32 or int64 [tokens], or [tokens,
    axes] for a plan of several axes.  out may be x."""
    dtype, dev, shape = x.dtype, x.get_device(), x.shape
    dt = _FLOAT16.get(dtype)
    xs = x.stride()
    if dt is None or len(shape) != 3 or dev < 0 or (xs[2] != 1 and shape[2] > 1):
        raise ValueError("x: expected a bf16 or fp16 [tokens, heads, head_dim] CUDA tensor with contiguous heads")
    T, H, D = shape
    pairs, turns, layout = plan.axis_pairs, plan.turns, _LAYOUTS.get(plan.layout)
    axes = len(pairs)
    ps, pdt, pst = positions.shape, positions.dtype, positions.stride()
    if ((pdt is not torch.int32 and pdt is not torch.int64) or positions.get_device() != dev
            or not (ps == (T, axes) or (axes == 1 and ps == (T,)))):
        raise ValueError(f"positions: expected int32 or int64 [{T}, {axes}] on cuda:{dev}")
    if turns.dtype is not torch.int64 or turns.dim() != 1 or not turns.is_contiguous() or turns.get_device() != dev:
        raise ValueError(f"plan.turns: expected a contiguous int64 vector on cuda:{dev}")
    if not 1 <= axes <= 4 or layout is None:
        raise ValueError("plan: one to four axes, layout 'interleaved' or 'half'")
    if out is None:
        out = _empty((T, H, D), dtype, x.device, stream)
    os_ = out.stride()
    if out.dtype is not dtype or out.shape != shape or out.get_device() != dev or (os_[2] != 1 and D > 1):
        raise ValueError(f"out: expected a {dtype} {list(shape)} tensor on cuda:{dev} with contiguous heads")
    _check(_library().packed.qlin_rope(_pack_rope(
        x.data_ptr(), out.data_ptr(), xs[0], xs[1], os_[0], os_[1], T, H,
        positions.data_ptr(), pst[0], pst[1] if len(pst) == 2 else 0,
        turns.data_ptr(), plan.magnitude, D, 2 * turns.numel(), 64 if pdt is torch.int64 else 32,
        axes, *pairs, *(0,) * (4 - axes), layout, 1 if inverse else 0, dt), _stream(stream)), "qlin_rope")
    return out


# ------------------------------------------------------ a serving step ---

@dataclass
class FP8BlockTensor:
    """FP8 operand [rows, K] with a scale for each block of block_rows rows (1: activations,
    128: weights) and 128 elements of K."""
    codes: torch.Tensor          # uint8 [rows, K]
    scales: torch.Tensor         # float32 [ceil(K / 128), ceil(rows / block_rows)]
    rows: int
    K: int
    block_rows: int

    def desc(self) -> FP8BlockDesc:
        return FP8BlockDesc(self.codes.data_ptr(), self.scales.data_ptr(), self.rows, self.K, self.block_rows)


def qlin_fp8_block_scales(rows: int, K: int, block_rows: int) -> int:
    return _library().qlin_fp8_block_scales(rows, K, block_rows)


def alloc_fp8_block(rows: int, K: int, block_rows: int = 1, device="cuda", stream=None) -> FP8BlockTensor:
    if qlin_fp8_block_scales(rows, K, block_rows) == 0:
        raise ValueError(f"invalid block-scaled FP8 shape [{rows}, {K}], block_rows {block_rows}")
    return FP8BlockTensor(_empty((rows, K), torch.uint8, device, stream),
                          _empty(((K + 127) // 128, -(-rows // block_rows)), torch.float32, device, stream),
                          rows, K, block_rows)


def _fp8_block_on(q, name, dev) -> bytes:
    """The packed descriptor of a block-scaled FP8 operand whose tensors hold what it says,
    on device `dev`."""
    codes, scales, rows, K, br = q.codes, q.scales, q.rows, q.K, q.block_rows
    cs, ss = codes.shape, scales.shape
    if (codes.dtype is not torch.uint8 or len(cs) != 2 or cs[0] != rows or cs[1] != K or codes.get_device() != dev
            or not codes.is_contiguous()):
        raise ValueError(f"{name}.codes: expected a contiguous uint8 [{rows}, {K}] tensor on cuda:{dev}")
    if ((br != 1 and br != 128) or scales.dtype is not torch.float32 or len(ss) != 2 or ss[0] != (K + 127) // 128
            or ss[1] != -(-rows // br) or scales.get_device() != dev or not scales.is_contiguous()):
        raise ValueError(f"{name}.scales: expected a contiguous float32 [ceil(K / 128), ceil(rows / block_rows)] "
                         f"tensor on cuda:{dev}, block_rows 1 or 128")
    return _pack_fp8_block(codes.data_ptr(), scales.data_ptr(), rows, K, br)


def qlin_quantize_fp8_block(x: torch.Tensor, block_rows: int = 1, out: FP8BlockTensor | None = None,
                            stream=None) -> FP8BlockTensor:
    """x [rows, K] (bf16 or fp16, rows any multiple of 8 elements apart) as a block-scaled
    FP8 operand; block_rows as in ``out`` where that is given."""
    dtype, dev, shape = x.dtype, x.get_device(), x.shape
    dt = _FLOAT16.get(dtype)
    if dt is None or len(shape) != 2 or dev < 0:
        raise ValueError("x: expected a 2-D bf16 or fp16 CUDA tensor")
    rows, K = shape
    stride = _rows16(x, "x", dtype, rows, K, dev)
    if out is None:
        out = alloc_fp8_block(rows, K, block_rows, x.device, stream)
    elif out.rows != rows or out.K != K:
        raise ValueError(f"out: expected an operand [{rows}, {K}]")
    _check(_library().packed.qlin_quantize_fp8_block(x.data_ptr(), dt, stride, _fp8_block_on(out, "out", dev),
                                                     _stream(stream)), "qlin_quantize_fp8_block")
    return out


def qlin_linear_fp8_block(A: FP8BlockTensor, W: FP8BlockTensor, bias: torch.Tensor | None = None,
                          act: int = QLIN_ACT_NONE, residual: torch.Tensor | None = None,
                          y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = act(A W^T + bias) + residual (bf16, one rounding) of block-scaled FP8 operands, A
    with block_rows 1 and W with 128.  residual may be y."""
    M, N, codes = A.rows, W.rows, A.codes
    dev = codes.get_device()
    if dev < 0:
        raise ValueError("A: expected a CUDA operand")
    ad, wd = _fp8_block_on(A, "A", dev), _fp8_block_on(W, "W", dev)
    if y is None:
        y = _empty((M, N), torch.bfloat16, codes.device, stream)
    yp = _dense16(y, "y", torch.bfloat16, M, N, dev)
    _check(_library().packed.qlin_linear_fp8_block(ad, wd, _epilogue(bias, act, residual, torch.bfloat16, M, N, dev),
                                                   yp, _stream(stream)), "qlin_linear_fp8_block")
    return y


_CACHE_FORMATS = {torch.bfloat16: QLIN_CACHE_BF16, torch.float16: QLIN_CACHE_FP16,
                  torch.float8_e4m3fn: QLIN_CACHE_E4M3}


@dataclass
class PagedCache:
    """Keys and values in pages, and a step's sequences: token i of sequence b, cached ones
    first, lies in page page_table[b, i // page_size], slot i % page_size; its new tokens are
    q_start[b] .. q_start[b + 1] - 1 of the call's."""
    k: torch.Tensor              # bf16, fp16 or float8_e4m3fn [pages, page_size, heads, head_dim]
    v: torch.Tensor
    page_table: torch.Tensor     # int32 [sequences, table_width]
    cached: torch.Tensor         # int32 [sequences]
    q_start: torch.Tensor        # int32 [sequences + 1]
    k_scale: torch.Tensor | None = None   # float32 [1], float8_e4m3fn only
    v_scale: torch.Tensor | None = None


def _cache_on(c, dev):
    """(the packed descriptor of a cache on device `dev`, heads, head_dim)."""
    k, v, table, cached, q_start = c.k, c.v, c.page_table, c.cached, c.q_start
    shape, fmt = k.shape, _CACHE_FORMATS.get(k.dtype)
    ks, vs = k.stride(), v.stride()
    if (fmt is None or len(shape) != 4 or v.dtype is not k.dtype or v.shape != shape or k.get_device() != dev
            or v.get_device() != dev or (shape[3] > 1 and (ks[3] != 1 or vs[3] != 1))):
        raise ValueError("cache: expected k and v bf16, fp16 or float8_e4m3fn [pages, page_size, heads, head_dim] "
                         f"on cuda:{dev} with contiguous heads")
    cs, qs, ts, tst, i32 = cached.shape, q_start.shape, table.shape, table.stride(), torch.int32
    if len(cs) != 1 or cached.dtype is not i32 or cached.get_device() != dev or not cached.is_contiguous():
        raise ValueError(f"cache.cached: expected a contiguous int32 vector on cuda:{dev}")
    B = cs[0]
    if (len(qs) != 1 or qs[0] != B + 1 or q_start.dtype is not i32 or q_start.get_device() != dev
            or not q_start.is_contiguous()):
        raise ValueError(f"cache.q_start: expected a contiguous int32 [{B + 1}] tensor on cuda:{dev}")
    if (len(ts) != 2 or ts[0] != B or table.dtype is not i32 or table.get_device() != dev
            or (tst[1] != 1 and ts[1] > 1)):
        raise ValueError(f"cache.page_table: expected an int32 [{B}, table_width] tensor on cuda:{dev} with "
                         "contiguous rows")
    if fmt == QLIN_CACHE_E4M3:
        if c.k_scale is None or c.v_scale is None:
            raise ValueError("cache: an FP8 cache needs k_scale and v_scale")
        sk, sv = _scalar32(c.k_scale, "cache.k_scale", dev), _scalar32(c.v_scale, "cache.v_scale", dev)
    else:
        sk = sv = 0
    desc = _pack_cache(k.data_ptr(), v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], table.data_ptr(),
                       tst[0] if B > 1 else ts[1], cached.data_ptr(), q_start.data_ptr(), sk, sv, B,
                       shape[0], shape[1], ts[1], shape[2], shape[3], fmt)
    return desc, shape[2], shape[3]


def _heads16(t, name, dtype, T, H, D, dev):
    """The strides of a 16-bit [tokens, heads, head_dim] tensor with contiguous heads."""
    s, shape = t.stride(), t.shape
    if (t.dtype is not dtype or len(shape) != 3 or shape[0] != T or shape[1] != H or shape[2] != D
            or t.get_device() != dev or (s[2] != 1 and D > 1)):
        raise ValueError(f"{name}: expected a {dtype} [{T}, {H}, {D}] tensor on cuda:{dev} with contiguous heads")
    return s[0], s[1]


def qlin_cache_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, plan: RopePlan | None = None,
                      positions: torch.Tensor | None = None, q: torch.Tensor | None = None,
                      q_out: torch.Tensor | None = None, stream=None):
    """Writes the step's keys (rotated) and values to their slots in the cache and returns q
    rotated (in q_out, allocated where it is None; None without q).  k, v [tokens, heads,
    head_dim] and q [tokens, q_heads, head_dim] may be views of a QKV output.  positions: int32
    or int64 [tokens] or [tokens, axes]; None: each token's number in its sequence.  plan None:
    nothing turns.  q_out may be q."""
    dtype, dev, shape = k.dtype, k.get_device(), k.shape
    dt = _FLOAT16.get(dtype)
    if dt is None or len(shape) != 3 or dev < 0:
        raise ValueError("k: expected a bf16 or fp16 [tokens, heads, head_dim] CUDA tensor")
    desc, H, D = _cache_on(cache, dev)
    T = shape[0]
    ks, vs = _heads16(k, "k", dtype, T, H, D, dev), _heads16(v, "v", dtype, T, H, D, dev)
    qp, qop, Hq, qs, qos = 0, 0, 0, (0, 0), (0, 0)
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q: expected a [tokens, q_heads, head_dim] tensor")
        Hq = q.shape[1]
        qs, qp = _heads16(q, "q", dtype, T, Hq, D, dev), q.data_ptr()
        if q_out is None:
            q_out = _empty((T, Hq, D), dtype, q.device, stream)
        qos, qop = _heads16(q_out, "q_out", dtype, T, Hq, D, dev), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    pp, pst, bits, tp, mag, R, pairs, layout = 0, (0, 0), 32, 0, 1.0, 0, (), 0
    if plan is None:
        if positions is not None:
            raise ValueError("positions without a plan")
    else:
        turns, pairs, layout = plan.turns, plan.axis_pairs, _LAYOUTS.get(plan.layout)
        if turns.dtype is not torch.int64 or turns.dim() != 1 or not turns.is_contiguous() or turns.get_device() != dev:
            raise ValueError(f"plan.turns: expected a contiguous int64 vector on cuda:{dev}")
        if not 1 <= len(pairs) <= 4 or layout is None:
            raise ValueError("plan: one to four axes, layout 'interleaved' or 'half'")
        tp, mag, R = turns.data_ptr(), plan.magnitude, 2 * turns.numel()
        if positions is not None:
            pdt, ps = positions.dtype, positions.shape
            if ((pdt is not torch.int32 and pdt is not torch.int64) or positions.get_device() != dev
                    or not (ps == (T, len(pairs)) or (len(pairs) == 1 and ps == (T,)))):
                raise ValueError(f"positions: expected int32 or int64 [{T}, {len(pairs)}] on cuda:{dev}")
            st = positions.stride()
            pp, pst, bits = positions.data_ptr(), (st[0], st[1] if len(st) == 2 else 0), 64 if pdt is torch.int64 else 32
    _check(_library().packed.qlin_cache_append(desc, _pack_append(
        k.data_ptr(), v.data_ptr(), qp, qop, *ks, *vs, *qs, *qos, T, pp, *pst, tp, mag, Hq, R, bits, len(pairs),
        *pairs, *(0,) * (4 - len(pairs)), layout, dt), _stream(stream)), "qlin_cache_append")
    return q_out


def qlin_cache_attention_workspace_size() -> int:
    return _library().qlin_cache_attention_workspace_size()


def _zero_counters(size, dtype, device):
    """A workspace for one call: the library wants its first 8192 bytes zero."""
    t = torch.empty(size, dtype=dtype, device=device)
    t[:8192].zero_()
    return t


def alloc_cache_attention_workspace(device="cuda") -> torch.Tensor:
    return torch.zeros(qlin_cache_attention_workspace_size(), dtype=torch.uint8, device=device)


def qlin_cache_attention(cache: PagedCache, q: torch.Tensor, scale: float, mask: torch.Tensor | None = None,
                         out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Attention of the step's tokens q [tokens, q_heads, head_dim] over their sequences' keys
    in the cache (the new ones appended before).  mask: int64 words (uint64's bits) [tokens,
    words], bit i of a token's row saying whether it sees its sequence's new token i; None:
    those up to itself.  lse: float32 [tokens, q_heads], written where it is given.  out may
    be q.  Calls that overlap on the GPU must not share a workspace."""
    dtype, dev, shape = q.dtype, q.get_device(), q.shape
    dt = _FLOAT16.get(dtype)
    if dt is None or len(shape) != 3 or dev < 0:
        raise ValueError("q: expected a bf16 or fp16 [tokens, q_heads, head_dim] CUDA tensor")
    desc, H, D = _cache_on(cache, dev)
    T, Hq = shape[0], shape[1]
    qs = _heads16(q, "q", dtype, T, Hq, D, dev)
    if out is None:
        out = _empty((T, Hq, D), dtype, q.device, stream)
    os_ = _heads16(out, "out", dtype, T, Hq, D, dev)
    mp, ms, words, lp = 0, 0, 0, 0
    if mask is not None:
        if (mask.dtype is not torch.int64 or mask.dim() != 2 or mask.shape[0] != T or mask.get_device() != dev
                or (mask.stride(1) != 1 and mask.shape[1] > 1)):
            raise ValueError(f"mask: expected an int64 [{T}, words] tensor on cuda:{dev} with contiguous rows")
        mp, ms, words = mask.data_ptr(), mask.stride(0), mask.shape[1]
    if lse is not None:
        if (lse.dtype is not torch.float32 or lse.shape != (T, Hq) or lse.get_device() != dev
                or not lse.is_contiguous()):
            raise ValueError(f"lse: expected a contiguous float32 [{T}, {Hq}] tensor on cuda:{dev}")
        lp = lse.data_ptr()
    if workspace is None:
        workspace = _empty(qlin_cache_attention_workspace_size(), torch.uint8, q.device, stream, _zero_counters)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on cuda:{dev}")
    _check(_library().packed.qlin_cache_attention(desc, _pack_attention(
        q.data_ptr(), out.data_ptr(), lp, mp, *qs, *os_, ms, T, scale, Hq, words, dt), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream(stream)), "qlin_cache_attention")
    return out


def qlin_sync_status(stream=None) -> int:
    """Synchronise `stream`; return (and clear) the device status code."""
    return _library().qlin_sync_status(_stream(stream))


def qlin_selftest_bounded_wait(timeout_ns: int, stream=None) -> None:
    _check(_library().qlin_selftest_bounded_wait(timeout_ns, _stream(stream)),
           "qlin_selftest_bounded_wait")


def qlin_set_wait_timeout_ns(ns: int) -> None:
    _library().qlin_set_wait_timeout_ns(ns)


def qlin_status_str(status: int) -> str:
    return _library().qlin_status_str(status).decode()


def qlin_last_error() -> str:
    return _library().qlin_last_error().decode()
