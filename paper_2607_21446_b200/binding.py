"""Thin ctypes binding over libkroquant.so (include/kroquant.h).

Argument marshalling only: every step of the quantizer runs in the CUDA
kernels behind the C ABI.  torch is used for device memory and streams.  There
is no CPU fallback: if the library cannot be loaded, or a call returns a
non-zero status, a :class:`KroQuantError` is raised.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import os
import struct
import threading
from typing import Optional

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libkroquant.so")

KQ_OK = 0
PATHS = {"auto": 0, "tensor": 1, "alu": 2, "onchip": 3}
EXPORTS = [
    "kroquant_factors_create", "kroquant_factors_create_lu", "kroquant_factors_create_dense",
    "kroquant_factors_destroy", "kroquant_quantize_ex", "kroquant_transform_f32_ex",
    "kroquant_scale_quantize_ex", "kroquant_mxfp4_quantize_ex", "kroquant_quantize_dual",
    "kroquant_fwht_quantize", "kroquant_fwht_transform_f32",
    "kroquant_factors_get", "kroquant_factors_n_sets", "kroquant_quantize", "kroquant_quantize_host",
    "kroquant_quantize_path", "kroquant_dequantize", "kroquant_scale_quantize",
    "kroquant_mxfp4_quantize", "kroquant_transform_f32", "kroquant_debug_e2m1_codes",
    "kroquant_tuning_default", "kroquant_quantize_tuned", "kroquant_quantize_dual_tuned", "kroquant_transform_f32_tuned",
    "kroquant_scale_quantize_tuned", "kroquant_mxfp4_quantize_tuned", "kroquant_fwht_quantize_tuned", "kroquant_debug_set_timeline", "kroquant_debug_withhold_arrival", "kroquant_debug_boundary_probe", "kroquant_launch_count", "kroquant_last_device_error",
    "kroquant_status_string",
    "kroquant_epilogue_default", "kroquant_linear_mxfp4", "kroquant_linear_mxfp4_grouped", "kroquant_norm_args_default",
    "kroquant_norm_residual", "kroquant_norm_residual_grad", "kroquant_norm_residual_grad_scratch_bytes",
    "kroquant_calib_create", "kroquant_calib_destroy", "kroquant_calib_set_theta", "kroquant_calib_get_theta",
    "kroquant_calib_set_lambdas", "kroquant_calib_get_lambdas", "kroquant_calib_get_factors",
    "kroquant_calib_loss_grad", "kroquant_calib_run",
    "kroquant_block_grad_scratch_bytes", "kroquant_block_grad", "kroquant_block_grad_static",
    "kroquant_calib_set_gemm_variant", "kroquant_gemm_mxfp4_variant", "kroquant_gemm_bf16_variant", "kroquant_calib_get_weight_factors", "kroquant_gemm_mxfp4",
    "kroquant_linear_w4a4", "kroquant_gemm_bf16",
    "kroquant_rotary_args_default", "kroquant_rotary", "kroquant_cache_write", "kroquant_cache_read",
    "kroquant_cache_attention_scratch_bytes", "kroquant_cache_attention", "kroquant_linear_w4a16",
]


class KroQuantError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


_lib: Optional[C.CDLL] = None


def load_library() -> C.CDLL:
    """Load libkroquant.so (built in-tree by ``paper_2607_21446_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2607_21446_b200.build` "
            "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    L.kroquant_factors_create.argtypes = [vp, i32, C.POINTER(vp)]
    L.kroquant_factors_create_lu.argtypes = [vp, i32, C.POINTER(vp)]
    L.kroquant_factors_create_dense.argtypes = [vp, i32, C.POINTER(vp)]
    L.kroquant_quantize_ex.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, i32, vp]
    L.kroquant_transform_f32_ex.argtypes = [vp, i32, i64, i32, vp, vp, i32, vp]
    L.kroquant_quantize_dual.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, vp, vp]
    L.kroquant_fwht_quantize.argtypes = [vp, i32, i64, i32, vp, vp, vp]
    L.kroquant_fwht_transform_f32.argtypes = [vp, i32, i64, i32, vp, vp]
    L.kroquant_scale_quantize_ex.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, vp]
    L.kroquant_mxfp4_quantize_ex.argtypes = [vp, i32, i64, i32, vp, vp, i32, vp]
    L.kroquant_factors_destroy.argtypes = [vp]
    L.kroquant_factors_destroy.restype = None
    L.kroquant_factors_get.argtypes = [vp, vp]
    L.kroquant_factors_n_sets.argtypes = [vp]
    L.kroquant_quantize.argtypes = [vp, i64, i32, vp, vp, vp, vp]
    L.kroquant_quantize_path.argtypes = [vp, i64, i32, vp, vp, vp, i32, vp]
    L.kroquant_quantize_host.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp, vp, vp]
    L.kroquant_dequantize.argtypes = [vp, vp, i64, i32, vp, vp, i32, vp]
    L.kroquant_scale_quantize.argtypes = [vp, i64, i32, vp, vp, vp, vp]
    L.kroquant_mxfp4_quantize.argtypes = [vp, i64, i32, vp, vp, vp]
    L.kroquant_transform_f32.argtypes = [vp, i64, i32, vp, vp, i32, vp]
    L.kroquant_debug_e2m1_codes.argtypes = [vp, i64, vp, vp]
    L.kroquant_debug_withhold_arrival.argtypes = [i32]
    L.kroquant_tuning_default.argtypes = [vp]
    L.kroquant_tuning_default.restype = None
    L.kroquant_quantize_tuned.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, i32, vp, vp]
    L.kroquant_quantize_dual_tuned.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, vp, vp, vp]
    L.kroquant_transform_f32_tuned.argtypes = [vp, i32, i64, i32, vp, vp, i32, vp, vp]
    L.kroquant_scale_quantize_tuned.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, vp, vp]
    L.kroquant_mxfp4_quantize_tuned.argtypes = [vp, i32, i64, i32, vp, vp, i32, vp, vp]
    L.kroquant_fwht_quantize_tuned.argtypes = [vp, i32, i64, i32, vp, vp, vp, vp]
    L.kroquant_debug_set_timeline.argtypes = [vp]
    L.kroquant_debug_boundary_probe.argtypes = [i32, i32, i32, i32, i32, vp, vp]
    L.kroquant_launch_count.argtypes = []
    L.kroquant_launch_count.restype = i64
    L.kroquant_last_device_error.argtypes = [vp, C.POINTER(i32)]
    L.kroquant_status_string.argtypes = [i32]
    L.kroquant_status_string.restype = C.c_char_p
    L.kroquant_calib_create.argtypes = [vp, vp, i64, i32, i32, i32, vp, C.POINTER(vp)]
    L.kroquant_calib_destroy.argtypes = [vp]
    L.kroquant_calib_destroy.restype = None
    for name in ("set_theta", "get_theta", "set_lambdas", "get_lambdas", "get_factors", "get_weight_factors"):
        getattr(L, "kroquant_calib_" + name).argtypes = [vp, vp]
    L.kroquant_calib_loss_grad.argtypes = [vp, vp, vp, vp]
    L.kroquant_calib_run.argtypes = [vp, i32, C.c_float, vp, vp]
    L.kroquant_block_grad_scratch_bytes.argtypes = [i64, i32]
    L.kroquant_block_grad_scratch_bytes.restype = i64
    L.kroquant_block_grad.argtypes = [vp, vp, i64, i32, i32, vp, i64, vp, vp]
    L.kroquant_block_grad_static.argtypes = [vp, vp, i64, i32, i32, vp, vp]
    L.kroquant_calib_set_gemm_variant.argtypes = [vp, i32]
    L.kroquant_gemm_mxfp4_variant.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, i32, i32, vp]
    L.kroquant_gemm_bf16_variant.argtypes = [vp, vp, i64, i32, i32, vp, vp, i32, i32, vp]
    L.kroquant_gemm_mxfp4.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, i32, vp]
    L.kroquant_gemm_bf16.argtypes = [vp, vp, i64, i32, i32, vp, vp, i32, vp]
    L.kroquant_linear_w4a4.argtypes = [vp, i32, i64, i32, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp]
    L.kroquant_epilogue_default.argtypes = [vp]
    L.kroquant_epilogue_default.restype = None
    L.kroquant_linear_mxfp4.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, i32, i64, vp]
    L.kroquant_linear_mxfp4_grouped.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, i32, vp, vp, i32, i64, vp]
    L.kroquant_norm_args_default.argtypes = [vp]
    L.kroquant_norm_args_default.restype = None
    L.kroquant_norm_residual.argtypes = [vp, vp]
    L.kroquant_norm_residual_grad_scratch_bytes.argtypes = [vp]
    L.kroquant_norm_residual_grad_scratch_bytes.restype = i64
    L.kroquant_norm_residual_grad.argtypes = [vp, vp, i64, vp]
    L.kroquant_rotary_args_default.argtypes = [vp]
    L.kroquant_rotary_args_default.restype = None
    L.kroquant_rotary.argtypes = [vp, vp]
    L.kroquant_cache_write.argtypes = [vp, vp, vp]
    L.kroquant_cache_read.argtypes = [vp, vp, vp]
    L.kroquant_cache_attention_scratch_bytes.argtypes = [vp, vp]
    L.kroquant_cache_attention_scratch_bytes.restype = i64
    L.kroquant_cache_attention.argtypes = [vp, vp, vp, i64, vp]
    L.kroquant_linear_w4a16.argtypes = [vp, i32, i64, vp, vp, i64, i32, i32, vp, vp, i32, i64, vp]
    _lib = L
    return L


def status_string(status: int) -> str:
    return load_library().kroquant_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != KQ_OK:
        raise KroQuantError(status, where)


# the handle itself where torch offers it: building a Stream object around it takes 4 us of a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", torch.cuda.is_current_stream_capturing)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


_CURRENT = contextlib.nullcontext()


def _allocating(stream):
    """Context in which outputs and scratch space are allocated for a call on `stream`: that stream's, so that the memory is
    neither still in use by another stream nor handed on before the call has run."""
    if stream is None:
        return _CURRENT
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


def _empty_rows(like: torch.Tensor, dtype, stream) -> torch.Tensor:
    """A tensor of like's shape with rows one after the other (empty_like costs 1 us of a call, new_empty with a shape 2)."""
    if stream is None:
        return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
    with _allocating(stream):
        return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


X_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
SCALE_LAYOUTS = {"rowmajor": 0, "tiled": 1}


def tiled_scale_bytes(tokens: int, d: int) -> int:
    """Size of the scale buffer in the 128 x 4 tiled layout."""
    return ((tokens + 127) // 128) * 128 * (((d // 32) + 3) // 4) * 4


def _scale_buffer(tokens: int, d: int, layout: str, device) -> torch.Tensor:
    if layout == "tiled":      # padding bytes are never written by the kernels: start from zeros
        return torch.zeros(tiled_scale_bytes(tokens, d), dtype=torch.uint8, device=device)
    return torch.empty((tokens, max(d // 32, 0)), dtype=torch.uint8, device=device)


def _x_shape(X: torch.Tensor) -> tuple[int, int]:
    if X.dim() != 2 or X.dtype not in X_DTYPES or not X.is_cuda or not X.is_contiguous():
        raise ValueError("X must be a contiguous 2-D CUDA bfloat16 or float16 tensor [tokens, d]")
    return X.shape[0], X.shape[1]


class Factors:
    """Handle of a kroquant_factors_t.  G: float32 [n_sets, 5, 2, 2] (host)."""

    def __init__(self, handle: int, n_sets: int):
        self._h = C.c_void_p(handle)
        self.n_sets = n_sets

    @classmethod
    def create(cls, G) -> "Factors":
        G = np.ascontiguousarray(G, dtype=np.float32)
        if G.ndim != 4 or G.shape[1:] != (5, 2, 2):
            raise ValueError("G must have shape [n_sets, 5, 2, 2]")
        out = C.c_void_p()
        _check(load_library().kroquant_factors_create(G.ctypes.data_as(C.c_void_p), G.shape[0],
                                                      C.byref(out)), "kroquant_factors_create")
        return cls(out.value, G.shape[0])

    @classmethod
    def create_lu(cls, abc) -> "Factors":
        abc = np.ascontiguousarray(abc, dtype=np.float32)
        if abc.ndim != 3 or abc.shape[1:] != (5, 3):
            raise ValueError("abc must have shape [n_sets, 5, 3]")
        out = C.c_void_p()
        _check(load_library().kroquant_factors_create_lu(abc.ctypes.data_as(C.c_void_p), abc.shape[0],
                                                         C.byref(out)), "kroquant_factors_create_lu")
        return cls(out.value, abc.shape[0])

    @classmethod
    def create_dense(cls, K) -> "Factors":
        """K: float32 [n_sets, 32, 32] dense blocks, y = x K per block."""
        K = np.ascontiguousarray(K, dtype=np.float32)
        if K.ndim != 3 or K.shape[1:] != (32, 32):
            raise ValueError("K must have shape [n_sets, 32, 32]")
        out = C.c_void_p()
        _check(load_library().kroquant_factors_create_dense(K.ctypes.data_as(C.c_void_p), K.shape[0],
                                                            C.byref(out)), "kroquant_factors_create_dense")
        return cls(out.value, K.shape[0])

    def get(self) -> np.ndarray:
        G = np.empty((self.n_sets, 5, 2, 2), np.float32)
        _check(load_library().kroquant_factors_get(self._h, G.ctypes.data_as(C.c_void_p)),
               "kroquant_factors_get")
        return G

    def destroy(self) -> None:
        if self._h:
            load_library().kroquant_factors_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Tuning(C.Structure):
    """kq_tuning_t: per-call tuning of the quantizer kernels (see include/kroquant.h).  ``Tuning()`` holds the
    library's defaults; keyword arguments override single fields."""
    _fields_ = [(n, C.c_int) for n in ("config", "ctas_per_sm", "use_pdl", "trigger", "prefetch_tiles", "dynamic",
                                       "unit_tiles", "compare_staged")]

    def __init__(self, **kw):
        super().__init__()
        load_library().kroquant_tuning_default(C.byref(self))
        for k, v in kw.items():
            if k not in dict(self._fields_):
                raise TypeError(f"unknown tuning field {k}")
            setattr(self, k, int(v))


def _tuning(t: Optional["Tuning"]):
    return None if t is None else C.cast(C.pointer(t), C.c_void_p)


def kroquant_quantize(X: torch.Tensor, factors: Factors, q_packed: Optional[torch.Tensor] = None,
                      scales: Optional[torch.Tensor] = None, path: str = "auto", stream=None,
                      scale_layout: str = "rowmajor", tuning: Optional[Tuning] = None):
    """(X bf16/fp16 [tokens, d], factors) -> (q_packed uint8 [tokens, d/2], scales uint8 [tokens, d/32]
    or, with scale_layout="tiled", a flat uint8 buffer in the 128 x 4 tiled layout)."""
    tokens, d = _x_shape(X)
    if q_packed is None:
        q_packed = torch.empty((tokens, max(d // 2, 0)), dtype=torch.uint8, device=X.device)
    if scales is None:
        scales = _scale_buffer(tokens, d, scale_layout, X.device)
    _check(load_library().kroquant_quantize_tuned(_ptr(X), X_DTYPES[X.dtype], tokens, d, factors._h, _ptr(q_packed),
                                                  _ptr(scales), SCALE_LAYOUTS[scale_layout], PATHS[path], _tuning(tuning),
                                                  C.c_void_p(_stream(stream))),
           "kroquant_quantize")
    return q_packed, scales


def kroquant_quantize_dual(X: torch.Tensor, factors: Factors, q_packed=None, scales=None, AT=None, stream=None,
                           scale_layout: str = "rowmajor", tuning: Optional[Tuning] = None):
    """One pass: MXFP4(X T) and X T itself in X's dtype -> (q_packed, scales, AT)."""
    tokens, d = _x_shape(X)
    if q_packed is None:
        q_packed = torch.empty((tokens, d // 2), dtype=torch.uint8, device=X.device)
    if scales is None:
        scales = _scale_buffer(tokens, d, scale_layout, X.device)
    if AT is None:
        AT = torch.empty_like(X)
    _check(load_library().kroquant_quantize_dual_tuned(_ptr(X), X_DTYPES[X.dtype], tokens, d, factors._h, _ptr(q_packed),
                                                       _ptr(scales), SCALE_LAYOUTS[scale_layout], _ptr(AT), _tuning(tuning),
                                                       C.c_void_p(_stream(stream))), "kroquant_quantize_dual")
    return q_packed, scales, AT


def kroquant_fwht_quantize(X: torch.Tensor, q_packed=None, scales=None, stream=None, tuning: Optional[Tuning] = None):
    """Full-d Walsh-Hadamard comparison quantizer (d a power of two, 32..16384)."""
    tokens, d = _x_shape(X)
    if q_packed is None:
        q_packed = torch.empty((tokens, d // 2), dtype=torch.uint8, device=X.device)
    if scales is None:
        scales = torch.empty((tokens, d // 32), dtype=torch.uint8, device=X.device)
    _check(load_library().kroquant_fwht_quantize_tuned(_ptr(X), X_DTYPES[X.dtype], tokens, d, _ptr(q_packed), _ptr(scales),
                                                       _tuning(tuning), C.c_void_p(_stream(stream))), "kroquant_fwht_quantize")
    return q_packed, scales


def kroquant_fwht_transform_f32(X: torch.Tensor, Y=None, stream=None):
    tokens, d = _x_shape(X)
    if Y is None:
        Y = torch.empty((tokens, d), dtype=torch.float32, device=X.device)
    _check(load_library().kroquant_fwht_transform_f32(_ptr(X), X_DTYPES[X.dtype], tokens, d, _ptr(Y),
                                                      C.c_void_p(_stream(stream))), "kroquant_fwht_transform_f32")
    return Y


def kroquant_scale_quantize(X: torch.Tensor, s: torch.Tensor, q_packed=None, scales=None, stream=None,
                            scale_layout: str = "rowmajor", tuning: Optional[Tuning] = None):
    tokens, d = _x_shape(X)
    if s.dtype != torch.float32 or not s.is_cuda or s.numel() != d or not s.is_contiguous():
        raise ValueError("s must be a contiguous CUDA float32 tensor [d]")
    if q_packed is None:
        q_packed = torch.empty((tokens, d // 2), dtype=torch.uint8, device=X.device)
    if scales is None:
        scales = _scale_buffer(tokens, d, scale_layout, X.device)
    _check(load_library().kroquant_scale_quantize_tuned(_ptr(X), X_DTYPES[X.dtype], tokens, d, _ptr(s), _ptr(q_packed),
                                                        _ptr(scales), SCALE_LAYOUTS[scale_layout], _tuning(tuning),
                                                        C.c_void_p(_stream(stream))),
           "kroquant_scale_quantize")
    return q_packed, scales


def kroquant_mxfp4_quantize(X: torch.Tensor, q_packed=None, scales=None, stream=None,
                            scale_layout: str = "rowmajor", tuning: Optional[Tuning] = None):
    tokens, d = _x_shape(X)
    if q_packed is None:
        q_packed = torch.empty((tokens, d // 2), dtype=torch.uint8, device=X.device)
    if scales is None:
        scales = _scale_buffer(tokens, d, scale_layout, X.device)
    _check(load_library().kroquant_mxfp4_quantize_tuned(_ptr(X), X_DTYPES[X.dtype], tokens, d, _ptr(q_packed),
                                                        _ptr(scales), SCALE_LAYOUTS[scale_layout], _tuning(tuning),
                                                        C.c_void_p(_stream(stream))),
           "kroquant_mxfp4_quantize")
    return q_packed, scales


def kroquant_transform_f32(X: torch.Tensor, factors: Factors, Y=None, path: str = "auto", stream=None,
                           tuning: Optional[Tuning] = None):
    tokens, d = _x_shape(X)
    if Y is None:
        Y = torch.empty((tokens, d), dtype=torch.float32, device=X.device)
    _check(load_library().kroquant_transform_f32_tuned(_ptr(X), X_DTYPES[X.dtype], tokens, d, factors._h, _ptr(Y),
                                                       PATHS[path], _tuning(tuning), C.c_void_p(_stream(stream))),
           "kroquant_transform_f32")
    return Y


def kroquant_dequantize(q_packed: torch.Tensor, scales: torch.Tensor, factors: Optional[Factors] = None,
                        out_dtype=torch.float32, out=None, stream=None):
    tokens, half = q_packed.shape
    d = half * 2
    if out is None:
        out = torch.empty((tokens, d), dtype=out_dtype, device=q_packed.device)
    code = {torch.float32: 0, torch.bfloat16: 1}[out.dtype]
    _check(load_library().kroquant_dequantize(_ptr(q_packed), _ptr(scales), tokens, d,
                                              factors._h if factors is not None else None, _ptr(out), code,
                                              C.c_void_p(_stream(stream))), "kroquant_dequantize")
    return out


def kroquant_debug_e2m1_codes(v: torch.Tensor, stream=None) -> torch.Tensor:
    codes = torch.empty(v.numel(), dtype=torch.uint8, device=v.device)
    _check(load_library().kroquant_debug_e2m1_codes(_ptr(v), v.numel(), _ptr(codes),
                                                    C.c_void_p(_stream(stream))), "kroquant_debug_e2m1_codes")
    return codes


def use_library(path: str) -> None:
    """Load another build of the library (the timeline build) instead of libkroquant.so; call before anything else."""
    global LIB_PATH, _lib
    LIB_PATH, _lib = path, None


def kroquant_debug_boundary_probe(tmem_cols: int, ctas_per_sm: int, late_trigger: bool, spin_ns: int, calls: int,
                                  marks: torch.Tensor, stream=None) -> None:
    """Diagnostic build only: `calls` chained probe launches (see the header); marks: int64 [calls, 1024, 4] on the device."""
    assert marks.dtype == torch.int64 and marks.numel() >= calls * 1024 * 4 and marks.is_cuda
    _check(load_library().kroquant_debug_boundary_probe(tmem_cols, ctas_per_sm, 1 if late_trigger else 0, spin_ns, calls,
                                                        _ptr(marks), C.c_void_p(_stream(stream))), "kroquant_debug_boundary_probe")


def kroquant_debug_set_timeline(marks: Optional[torch.Tensor]) -> None:
    _check(load_library().kroquant_debug_set_timeline(_ptr(marks)), "kroquant_debug_set_timeline")


def kroquant_debug_withhold_arrival(on: bool) -> None:
    _check(load_library().kroquant_debug_withhold_arrival(int(on)), "kroquant_debug_withhold_arrival")


def kroquant_launch_count() -> int:
    return int(load_library().kroquant_launch_count())


def kroquant_last_device_error(stream=None) -> int:
    code = C.c_int(0)
    _check(load_library().kroquant_last_device_error(C.c_void_p(_stream(stream)), C.byref(code)),
           "kroquant_last_device_error")
    return int(code.value)


# ---- host-buffer convenience used for end-to-end timing -------------------------
def quantize_from_host(X_host: torch.Tensor, factors: Factors, X_dev: torch.Tensor, q_dev: torch.Tensor,
                       s_dev: torch.Tensor, q_host: torch.Tensor, s_host: torch.Tensor, stream=None):
    """Pinned host X -> device, quantize, codes + scales -> pinned host.  All async on `stream`."""
    X_dev.copy_(X_host, non_blocking=True)
    kroquant_quantize(X_dev, factors, q_dev, s_dev, stream=stream)
    q_host.copy_(q_dev, non_blocking=True)
    s_host.copy_(s_dev, non_blocking=True)
    return q_host, s_host


def kroquant_quantize_host(X_host: torch.Tensor, factors: Factors, q_host: torch.Tensor, s_host: torch.Tensor,
                           X_work: torch.Tensor, q_work: torch.Tensor, s_work: torch.Tensor, stream=None) -> None:
    """Host tensors in, host tensors out, through the caller's device work buffers: one C call that issues the
    upload, the kernel and the two downloads in order on `stream` (asynchronous when the host tensors are pinned)."""
    tokens, d = X_host.shape
    assert X_host.dtype == torch.bfloat16 and X_host.is_contiguous() and not X_host.is_cuda
    assert q_host.shape == (tokens, d // 2) and s_host.shape == (tokens, d // 32) and not q_host.is_cuda
    assert X_work.is_cuda and X_work.shape == X_host.shape and q_work.shape == q_host.shape and s_work.shape == s_host.shape
    _check(load_library().kroquant_quantize_host(
        C.c_void_p(X_host.data_ptr()), tokens, d, factors._h, C.c_void_p(q_host.data_ptr()), C.c_void_p(s_host.data_ptr()),
        C.c_void_p(X_work.data_ptr()), C.c_void_p(q_work.data_ptr()), C.c_void_p(s_work.data_ptr()), C.c_void_p(_stream(stream))),
        "kroquant_quantize_host")


def kroquant_block_grad(X: torch.Tensor, G: torch.Tensor, n_sets: int = 1, out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """out[s] = sum of x_j^T g_j over rows (and over block columns for a shared set): float32
    [n_sets, 32, 32].  X: CUDA bfloat16 [rows, d]; G: CUDA float32 [rows, d].  The scratch buffer the
    kernel needs is allocated here (torch) and passed down."""
    rows, d = _x_shape(X)
    if X.dtype != torch.bfloat16 or G.dtype != torch.float32 or G.shape != X.shape or not G.is_contiguous():
        raise ValueError("X bfloat16 [rows, d] and G float32 [rows, d], both contiguous")
    L = load_library()
    if out is None:
        out = torch.empty((n_sets, 32, 32), dtype=torch.float32, device=X.device)
    nbytes = max(int(L.kroquant_block_grad_scratch_bytes(rows, d)), 16)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=X.device)
    _check(L.kroquant_block_grad(_ptr(X), _ptr(G), rows, d, n_sets, _ptr(scratch), nbytes, _ptr(out), _stream(stream)),
           "kroquant_block_grad")
    return out


def kroquant_block_grad_static(X: torch.Tensor, G: torch.Tensor, n_sets: int, out: torch.Tensor, stream=None) -> None:
    """kroquant_block_grad without a scratch buffer: the library's built-in one is used, so nothing is
    allocated here or below (``out``, float32 [n_sets, 32, 32], must be supplied).  For callers whose
    device memory is spoken for; see the header for the size limit and the sharing rules."""
    rows, d = _x_shape(X)
    if X.dtype != torch.bfloat16 or G.dtype != torch.float32 or G.shape != X.shape or not G.is_contiguous():
        raise ValueError("X bfloat16 [rows, d] and G float32 [rows, d], both contiguous")
    if out.dtype != torch.float32 or tuple(out.shape) != (n_sets, 32, 32) or not out.is_contiguous() or not out.is_cuda:
        raise ValueError("out must be a contiguous CUDA float32 tensor [n_sets, 32, 32]")
    _check(load_library().kroquant_block_grad_static(_ptr(X), _ptr(G), rows, d, n_sets, _ptr(out), _stream(stream)),
           "kroquant_block_grad_static")


def kroquant_gemm_mxfp4(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor, b_scales: torch.Tensor,
                        add: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        out_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """out[M, N] = (codes, tiled scales of A [M, K]) x (codes, tiled scales of B [N, K])^T (+ add): the W4A4
    product on the block-scaled FP4 tensor-core path.  Inputs are what the quantizer calls return with
    ``scale_layout="tiled"``."""
    for t in (a_codes, a_scales, b_codes, b_scales):
        if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("codes and scales must be contiguous CUDA uint8 tensors")
    M, half = a_codes.shape
    N = b_codes.shape[0]
    if b_codes.shape[1] != half:
        raise ValueError("A and B must share K")
    K = 2 * half
    if a_scales.numel() != tiled_scale_bytes(M, K) or b_scales.numel() != tiled_scale_bytes(N, K):
        raise ValueError("scales must be in the tiled layout (tiled_scale_bytes(rows, K) bytes)")
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=a_codes.device)
    if out.dtype not in (torch.bfloat16, torch.float32) or tuple(out.shape) != (M, N) or not out.is_contiguous():
        raise ValueError("out must be a contiguous bfloat16 or float32 tensor [M, N]")
    if add is not None and (add.dtype != torch.bfloat16 or tuple(add.shape) != (M, N) or not add.is_contiguous()):
        raise ValueError("add must be a contiguous bfloat16 tensor [M, N]")
    _check(load_library().kroquant_gemm_mxfp4_variant(_ptr(a_codes), _ptr(a_scales), _ptr(b_codes), _ptr(b_scales), M, N, K,
                                                      _ptr(add), _ptr(out), 1 if out.dtype == torch.bfloat16 else 0,
                                                      int(_GEMM_PAIR), _stream(stream)), "kroquant_gemm_mxfp4")
    return out


def kroquant_gemm_bf16(A: torch.Tensor, Bm: torch.Tensor, add: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """out[M, N] = A[M, K] @ Bm[N, K]^T (+ add, float32): bf16 operands, fp32 accumulation, on this library's
    tensor-core GEMM (for the 16-bit low-rank branch of the quantized layer)."""
    for t in (A, Bm):
        if t.dim() != 2 or t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("A and Bm must be contiguous 2-D CUDA bfloat16 tensors")
    M, K = A.shape
    N = Bm.shape[0]
    if Bm.shape[1] != K:
        raise ValueError("A [M, K] and Bm [N, K] must share K")
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=A.device)
    if out.dtype not in (torch.bfloat16, torch.float32) or tuple(out.shape) != (M, N) or not out.is_contiguous():
        raise ValueError("out must be a contiguous bfloat16 or float32 tensor [M, N]")
    if add is not None and (add.dtype != torch.float32 or tuple(add.shape) != (M, N) or not add.is_contiguous()):
        raise ValueError("add must be a contiguous float32 tensor [M, N]")
    _check(load_library().kroquant_gemm_bf16_variant(_ptr(A), _ptr(Bm), M, N, K, _ptr(add), _ptr(out),
                                                     1 if out.dtype == torch.bfloat16 else 0, int(_GEMM_PAIR),
                                                     _stream(stream)), "kroquant_gemm_bf16")
    return out


class LinearW4A4:
    """The quantized linear layer of Section 3.4: holds the activation factors, the offline-quantized
    weights (codes + tiled scales) and the work buffers for Q(X T); ``__call__`` runs quantizer + FP4 GEMM
    (two launches, nothing allocated after the first call on a stream for the largest number of tokens).  Calls
    on different streams and from different threads have work buffers of their own."""

    def __init__(self, factors: "Factors", w_codes: torch.Tensor, w_scales: torch.Tensor):
        self.factors, self.w_codes, self.w_scales = factors, w_codes, w_scales
        self.o, self.d = w_codes.shape[0], 2 * w_codes.shape[1]
        self._work = {}

    @classmethod
    def from_weights(cls, W: torch.Tensor, G_act, G_weight) -> "LinearW4A4":
        """W: CUDA bf16 [o, d]; G_act / G_weight: factor sets [n_sets, 5, 2, 2] of T and T^-T."""
        fw = Factors.create(G_weight)
        q, s = kroquant_quantize(W, fw, scale_layout="tiled")
        torch.cuda.current_stream().synchronize()
        fw.destroy()
        return cls(Factors.create(G_act), q, s)

    def _buffers(self, tokens: int, device, stream, handle: int):
        """Work buffers for Q(X T) of this many tokens: one pair for each stream and calling thread, as large as the largest call
        needed, since calls that may overlap must not share them.  A graph under capture gets its own, since it may run next to
        later calls.  Scale bytes that the quantizer leaves out must not be 0xFF: kept buffers start from zeros, a graph's where
        there are such bytes."""
        capturing = _capturing()
        key = (handle, threading.get_ident())
        work = None if capturing else self._work.get(key)
        if work is None or work[0].shape[0] < tokens:
            with _allocating(stream):
                make = torch.empty if capturing and tokens % 128 == 0 and self.d % 128 == 0 else torch.zeros
                work = (torch.empty((tokens, self.d // 2), dtype=torch.uint8, device=device),
                        make(tiled_scale_bytes(tokens, self.d), dtype=torch.uint8, device=device))
            if not capturing:
                self._work[key] = work
        return work

    def __call__(self, X: torch.Tensor, add: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 out_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
        tokens, d = _x_shape(X)
        if d != self.d:
            raise ValueError("X [tokens, d] does not match the weights")
        handle = _stream(stream)
        q, s = self._buffers(tokens, X.device, stream, handle)
        if out is None:
            out = torch.empty((tokens, self.o), dtype=out_dtype, device=X.device)
        _check(load_library().kroquant_linear_w4a4(
            _ptr(X), X_DTYPES[X.dtype], tokens, d, self.factors._h, _ptr(self.w_codes), _ptr(self.w_scales), self.o,
            _ptr(q), _ptr(s), _ptr(add), _ptr(out), 1 if out.dtype == torch.bfloat16 else 0, handle),
            "kroquant_linear_w4a4")
        return out

    def fused(self, X: torch.Tensor, *, stream=None, **epilogue) -> torch.Tensor:
        """The layer with its epilogue: quantizer, then :func:`kroquant_linear_mxfp4` with the keyword arguments given here
        (bias, activation, glu, gate, row_scale, residual, out, ...).  Two launches.  (Without an epilogue ``__call__`` is the
        faster one for many rows: 4608 x 3072 -> 12288 in 85 against 105 us.)"""
        tokens, d = _x_shape(X)
        if d != self.d:
            raise ValueError("X [tokens, d] does not match the weights")
        handle = _stream(stream)
        q, s = self._buffers(tokens, X.device, stream, handle)
        if q.shape[0] != tokens:
            q, s = q[:tokens], s[:tiled_scale_bytes(tokens, d)]
        kroquant_quantize(X, self.factors, q, s, stream=handle, scale_layout="tiled")
        return kroquant_linear_mxfp4(q, s, self.w_codes, self.w_scales, stream=stream, **epilogue)

    def few(self, X: torch.Tensor, *, stream=None, **epilogue) -> torch.Tensor:
        """The layer for a few rows (at most 64) whose activations are transformed but not quantized: X T in X's own type
        (:func:`kroquant_quantize_dual`), then :func:`kroquant_linear_w4a16` with the keyword arguments given here.  Two launches."""
        tokens, d = _x_shape(X)
        if d != self.d:
            raise ValueError("X [tokens, d] does not match the weights")
        if tokens > 64:
            raise ValueError("X has more than 64 rows: use fused")
        handle = _stream(stream)
        q, s = self._buffers(tokens, X.device, stream, handle)
        q, s = q[:tokens], s[:tiled_scale_bytes(tokens, d)]
        with _allocating(stream):
            turned = torch.empty_like(X)
        kroquant_quantize_dual(X, self.factors, q, s, turned, stream=handle, scale_layout="tiled")
        return kroquant_linear_w4a16(turned, self.w_codes, self.w_scales, stream=stream, **epilogue)


# ---- the transformer block around the W4A4 product -----------------------------------------------------------------
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
NORMS = {"none": 0, "rms": 1, "layer": 2}
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class _Epilogue(C.Structure):
    """kq_epilogue_t (include/kroquant.h)."""
    _fields_ = [("activation", C.c_int), ("glu", C.c_int), ("bias", C.c_void_p), ("bias_dtype", C.c_int), ("gate", C.c_void_p),
                ("gate_dtype", C.c_int), ("gate_stride", C.c_int64), ("rows_per_gate", C.c_int64), ("row_scale", C.c_void_p),
                ("residual", C.c_void_p), ("residual_dtype", C.c_int), ("ld_residual", C.c_int64), ("residual_scale", C.c_float)]


class _NormArgs(C.Structure):
    """kq_norm_args_t (include/kroquant.h)."""
    _fields_ = ([("rows", C.c_int64)] + [(n, C.c_int) for n in ("d", "norm", "post_norm", "stream_dtype", "branch_dtype", "vec_dtype")] +
                [("residual_scale", C.c_float), ("eps", C.c_float), ("rows_per_batch", C.c_int64)] +
                [(n, C.c_void_p) for n in ("gate", "post_weight", "weight", "scale", "shift")] +
                [(n, C.c_int64) for n in ("gate_stride", "scale_stride", "shift_stride")] +
                [(n, C.c_void_p) for n in ("x", "y", "h", "n")] + [(n, C.c_int64) for n in ("ld_x", "ld_y", "ld_h", "ld_n")] +
                [(n, C.c_void_p) for n in ("dn", "dh", "dx", "dy")] + [(n, C.c_int64) for n in ("ld_dn", "ld_dh", "ld_dx", "ld_dy")] +
                [(n, C.c_void_p) for n in ("dgate", "dpost_weight", "dweight", "dscale", "dshift")])


def interleave_glu(W_gate: torch.Tensor, W_value: torch.Tensor) -> torch.Tensor:
    """[F, K] gate and value weights (or [F] biases) -> the rows a gated layer stores: 32 gate rows, their 32 value rows, ...,
    the last block filled up with zeros; [64 * ceil(F / 32), K].  Quantize the result as the layer's weight."""
    if W_gate.shape != W_value.shape or W_gate.dtype != W_value.dtype:
        raise ValueError("W_gate and W_value must have the same shape and dtype")
    F, blocks = W_gate.shape[0], (W_gate.shape[0] + 31) // 32
    out = W_gate.new_zeros((2, blocks * 32) + tuple(W_gate.shape[1:]))
    out[0, :F], out[1, :F] = W_gate, W_value
    return out.view(2, blocks, 32, -1).transpose(0, 1).reshape((blocks * 64,) + tuple(W_gate.shape[1:]))


def _rows2d(t: torch.Tensor, shape, what: str) -> int:
    """Pitch of a tensor of this 2-D shape with contiguous rows on the current device."""
    if t.shape == shape and t.dtype in _DTYPES and t.get_device() == _device():
        if t.is_contiguous():
            return shape[1]
        rows, cols = shape
        if (cols <= 1 or t.stride(1) == 1) and (rows <= 1 or t.stride(0) >= cols):
            return t.stride(0) if rows > 1 else cols
    raise ValueError(f"{what} must be a float32, bfloat16 or float16 tensor {list(shape)} on the current CUDA device with "
                     "contiguous rows that do not overlap")


def _span(t: torch.Tensor):
    """First byte of t and the one behind its last."""
    base, count = t.data_ptr(), t.numel()
    if count and not t.is_contiguous():
        count = 1
        for n, s in zip(t.shape, t.stride()):
            count += (n - 1) * s
    return base, base + count * t.element_size()


def _meet(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two tensors may have a byte in common."""
    return _spans_meet(a, _span(a), b, _span(b))


def _spans_meet(a: torch.Tensor, a_span, b: torch.Tensor, b_span) -> bool:
    """The same with the spans known."""
    if a_span[1] <= b_span[0] or b_span[1] <= a_span[0] or a_span[0] == a_span[1] or b_span[0] == b_span[1]:
        return False
    return not _parts_of_rows(b_span[0] - a_span[0], a.element_size(), a.shape, a.stride(), b.element_size(), b.shape, b.stride())


@functools.lru_cache(maxsize=256)
def _parts_of_rows(ahead: int, a_size: int, a_shape, a_stride, b_size: int, b_shape, b_stride) -> bool:
    """Whether tensors whose spans overlap, the second `ahead` bytes behind the first, have no byte in common all the same, as different parts of the
    same packed rows: a byte of both would need offsets within the rows that differ by a multiple of the rows' step, and so on within the row."""
    def apart(ahead, a_steps, b_steps):
        a_wide, b_wide = (size + sum((n - 1) * step for step, n in steps) for size, steps in ((a_size, a_steps), (b_size, b_steps)))
        if ahead >= a_wide or -ahead >= b_wide:
            return True
        if not a_steps and not b_steps:
            return False
        step = max(a_steps + b_steps)[0]
        a_in, b_in = ([p for p in steps if p[0] != step] for steps in (a_steps, b_steps))
        a_wide, b_wide = (size + sum((n - 1) * s for s, n in steps) for size, steps in ((a_size, a_in), (b_size, b_in)))
        ahead %= step
        first, last = -((a_wide - 1 - ahead) // step), (ahead + b_wide - 1) // step                    # multiples of the step that offsets may differ by
        return last - first < 4 and all(apart(ahead - m * step, a_in, b_in) for m in range(first, last + 1))

    return apart(ahead, [(s * a_size, n) for n, s in zip(a_shape, a_stride) if n > 1 and s], [(s * b_size, n) for n, s in zip(b_shape, b_stride) if n > 1 and s])


def _linear(a_codes, a_scales, b_codes, b_scales, offsets, features, bias, activation, glu, gate, rows_per_gate, row_scale,
            residual, residual_scale, out, out_dtype, stream, ld_x=None):
    dev = _device()
    b_shape, grouped, quantized = b_codes.shape, offsets is not None, ld_x is None
    for t in (a_codes, a_scales, b_codes, b_scales) if quantized else (b_codes, b_scales):
        if t.dtype is not torch.uint8 or t.get_device() != dev or not t.is_contiguous():
            raise ValueError("codes and scales must be contiguous uint8 tensors on the current CUDA device")
    M, K = a_codes.shape if a_codes.dim() == 2 else (0, -1)
    if quantized:
        K *= 2
    if K < 0 or len(b_shape) != (3 if grouped else 2) or 2 * b_shape[-1] != K:
        raise ValueError("A is [M, K/2] codes, B [rows, K/2] ([experts, rows, K/2] in the grouped call) with the same K" if quantized else
                         "x is [M, K], B [rows, K/2] codes with the same K")
    R, experts = b_shape[-2], b_shape[0] if grouped else 1
    if (quantized and a_scales.numel() != tiled_scale_bytes(M, K)) or b_scales.numel() != experts * tiled_scale_bytes(R, K):
        raise ValueError("scales must be in the tiled layout (tiled_scale_bytes(rows, K) bytes, per expert for B)")
    N = (R // 2 if glu else R) if features is None else features
    if R != (64 * ((N + 31) // 32) if glu else N):
        raise ValueError("B must have `features` rows, or 64 * ceil(features / 32) interleaved rows with glu")
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    e = _Epilogue()
    e.activation, e.glu, e.rows_per_gate, e.residual_scale = act, 1 if glu else 0, 1, residual_scale
    if bias is not None:
        if bias.shape != ((experts, R) if grouped else (R,)) or bias.dtype not in _DTYPES or bias.get_device() != dev or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous CUDA floating tensor with one entry per row of B")
        e.bias, e.bias_dtype = bias.data_ptr(), _DTYPES[bias.dtype]
    if gate is not None:
        rows = 1 if gate.dim() == 1 else gate.shape[0]
        if gate.dim() not in (1, 2) or gate.shape[-1] != N or gate.dtype not in _DTYPES or gate.get_device() != dev or \
                (N > 1 and gate.stride(-1) != 1) or (rows > 1 and gate.stride(0) < N):
            raise ValueError("gate must be a CUDA floating tensor [N] or [batches, N] with contiguous rows")
        if rows_per_gate is None:
            if rows < 1 or M % rows:
                raise ValueError("M is not a multiple of the gate's rows: pass rows_per_gate")
            rows_per_gate = max(M // rows, 1)
        if rows_per_gate < 1 or rows * rows_per_gate < M:
            raise ValueError("gate has too few rows for rows_per_gate")
        e.gate, e.gate_dtype, e.gate_stride, e.rows_per_gate = gate.data_ptr(), _DTYPES[gate.dtype], gate.stride(0) if rows > 1 else 0, rows_per_gate
    if row_scale is not None:
        if row_scale.shape != (M,) or row_scale.dtype is not torch.float32 or row_scale.get_device() != dev or not row_scale.is_contiguous():
            raise ValueError("row_scale must be a contiguous CUDA float32 tensor [M]")
        e.row_scale = row_scale.data_ptr()
    if residual is not None:
        e.ld_residual = _rows2d(residual, (M, N), "residual")
        e.residual, e.residual_dtype = residual.data_ptr(), _DTYPES[residual.dtype]
    if out is None:
        if out_dtype not in _DTYPES:
            raise ValueError("out_dtype must be float32, bfloat16 or float16")
        if stream is None:
            out = torch.empty_strided((M, N), (N, 1), dtype=out_dtype, device=a_codes.device)
        else:
            with _allocating(stream):
                out = torch.empty_strided((M, N), (N, 1), dtype=out_dtype, device=a_codes.device)
        ld_out = N
    else:
        ld_out = _rows2d(out, (M, N), "out")
        if not quantized and _meet(out, a_codes):
            raise ValueError("out must not overlap x, which other parts of the call still read")
    if grouped:
        if offsets.dtype is not torch.int32 or offsets.shape != (experts + 1,) or offsets.get_device() != dev or not offsets.is_contiguous():
            raise ValueError("offsets must be a contiguous CUDA int32 tensor [experts + 1]")
        rc = load_library().kroquant_linear_mxfp4_grouped(
            a_codes.data_ptr(), a_scales.data_ptr(), b_codes.data_ptr(), b_scales.data_ptr(), offsets.data_ptr(), experts, M, N, K,
            C.addressof(e), out.data_ptr(), _DTYPES[out.dtype], ld_out, _stream(stream))
    elif quantized:
        rc = load_library().kroquant_linear_mxfp4(
            a_codes.data_ptr(), a_scales.data_ptr(), b_codes.data_ptr(), b_scales.data_ptr(), M, N, K, C.addressof(e), out.data_ptr(),
            _DTYPES[out.dtype], ld_out, _stream(stream))
    else:
        rc = load_library().kroquant_linear_w4a16(
            a_codes.data_ptr(), X_DTYPES[a_codes.dtype], ld_x, b_codes.data_ptr(), b_scales.data_ptr(), M, N, K, C.addressof(e), out.data_ptr(),
            _DTYPES[out.dtype], ld_out, _stream(stream))
    if rc:
        raise KroQuantError(rc, "kroquant_linear_mxfp4_grouped" if grouped else "kroquant_linear_mxfp4" if quantized else "kroquant_linear_w4a16")
    return out


def kroquant_linear_mxfp4(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor, b_scales: torch.Tensor, *,
                          features: Optional[int] = None, bias: Optional[torch.Tensor] = None, activation: str = "none",
                          glu: bool = False, gate: Optional[torch.Tensor] = None, rows_per_gate: Optional[int] = None,
                          row_scale: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                          residual_scale: float = 1.0, out: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16,
                          stream=None) -> torch.Tensor:
    """The W4A4 product with the layer's epilogue:

        out = residual_scale * residual + row_scale[:, None] * gate * act(A B^T + bias)

    A, B: codes and tiled scales as the quantizer writes them (``scale_layout="tiled"``).  With ``glu`` B's rows (and
    bias's entries) are interleaved by :func:`interleave_glu` and v = act(A B_g^T + bias_g) * (A B_v^T + bias_v);
    ``features`` then gives the number of output columns (default: half of B's rows).  activation: none, relu, silu,
    gelu (erf) or gelu_tanh; gate [N] or [batches, N] (row m uses row m // rows_per_gate; default: M / batches); row_scale
    float32 [M].  bias, gate, residual and out may each be float32, bfloat16 or float16; residual and out may have a row
    pitch, and out may be the residual.  fp32 inside, rounded once."""
    return _linear(a_codes, a_scales, b_codes, b_scales, None, features, bias, activation, glu, gate, rows_per_gate, row_scale,
                   residual, residual_scale, out, out_dtype, stream)


def kroquant_linear_mxfp4_grouped(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor, b_scales: torch.Tensor,
                                  offsets: torch.Tensor, *, features: Optional[int] = None, bias: Optional[torch.Tensor] = None,
                                  activation: str = "none", glu: bool = False, row_scale: Optional[torch.Tensor] = None,
                                  residual: Optional[torch.Tensor] = None, residual_scale: float = 1.0,
                                  out: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """:func:`kroquant_linear_mxfp4` with one weight per expert: rows offsets[e] .. offsets[e + 1] - 1 of A (sorted by expert,
    quantized once, not padded) meet b_codes[e] ([experts, rows, K/2]; b_scales: the experts' tiled buffers one after
    another).  offsets: CUDA int32 [experts + 1], read on the device; groups may be empty.  Rows outside
    [offsets[0], offsets[-1]) are not written.  bias: [experts, rows of B]; row_scale: the router's weight of each row."""
    if offsets is None:
        raise ValueError("offsets must be a contiguous CUDA int32 tensor [experts + 1]")
    return _linear(a_codes, a_scales, b_codes, b_scales, offsets, features, bias, activation, glu, None, None, row_scale, residual,
                   residual_scale, out, out_dtype, stream)


def kroquant_linear_w4a16(x: torch.Tensor, b_codes: torch.Tensor, b_scales: torch.Tensor, *, features: Optional[int] = None,
                          bias: Optional[torch.Tensor] = None, activation: str = "none", glu: bool = False,
                          gate: Optional[torch.Tensor] = None, rows_per_gate: Optional[int] = None,
                          row_scale: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                          residual_scale: float = 1.0, out: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16,
                          stream=None) -> torch.Tensor:
    """:func:`kroquant_linear_mxfp4` with rows that stay in 16 bits: x [M, K] bfloat16 or float16 (a row pitch is allowed),
    1 <= M <= 64, the weight and the keyword arguments as there.  For a few rows (a decode step, a conditioning vector)
    it reads what the quantized form reads and keeps the activations' digits.  out may be the residual, but must not overlap x."""
    if x.dtype not in X_DTYPES:
        raise ValueError("x must be bfloat16 or float16")
    if x.dim() != 2:
        raise ValueError("x must be [M, K]")
    if x.shape[0] > 64:
        raise ValueError("x has more than 64 rows: quantize it and use kroquant_linear_mxfp4")
    return _linear(x, None, b_codes, b_scales, None, features, bias, activation, glu, gate, rows_per_gate, row_scale, residual,
                   residual_scale, out, out_dtype, stream, _rows2d(x, x.shape, "x"))


def _norm_args(rows: int, d: int, norm: str, post_norm: str, residual_scale: float, eps: float, rows_per_batch, gate, post_weight,
               weight, scale, shift) -> "_NormArgs":
    """The arguments that forward and backward share: settings, parameter vectors and their strides."""
    a = _NormArgs()
    try:
        a.norm, a.post_norm = NORMS[norm], NORMS[post_norm]
    except KeyError:
        raise ValueError(f"norm and post_norm must be one of {sorted(NORMS)}") from None
    a.rows, a.d, a.residual_scale, a.eps = rows, d, residual_scale, eps
    batches, dtype, dev = 1, None, _device()
    for name, v in (("gate", gate), ("post_weight", post_weight), ("weight", weight), ("scale", scale), ("shift", shift)):
        if v is None:
            continue
        shape = v.shape
        if dtype is None:
            dtype = v.dtype
        batched = len(shape) == 2 and name != "weight" and name != "post_weight"
        if shape[-1:] != (d,) or (len(shape) != 1 and not batched) or v.dtype not in _DTYPES or v.get_device() != dev or \
                not (v.is_contiguous() or ((d <= 1 or v.stride(-1) == 1) and (not batched or shape[0] <= 1 or v.stride(0) >= d))):
            raise ValueError(f"{name} must be a CUDA floating tensor [d]" + ("" if "weight" in name else " or [batches, d] with contiguous rows"))
        if v.dtype is not dtype:
            raise ValueError("gate, post_weight, weight, scale and shift must share a dtype")
        setattr(a, name, v.data_ptr())
        if batched and shape[0] != 1:
            if batches != 1 and batches != shape[0]:
                raise ValueError("batched vectors must agree on the number of batches")
            batches = shape[0]
            # (a gradient keeps the shape of its vector, so one row of [1, d] counts as one vector for all rows)
            setattr(a, name + "_stride", v.stride(0))
    if dtype is not None:
        a.vec_dtype = _DTYPES[dtype]
    if batches == 1:
        rows_per_batch = rows or 1
    elif rows_per_batch is None:
        if batches < 1 or rows % batches:
            raise ValueError("rows is not a multiple of the batches: pass rows_per_batch")
        rows_per_batch = rows // batches or 1
    if rows_per_batch < 1 or rows > batches * rows_per_batch:
        raise ValueError("the batched vectors have too few rows for rows_per_batch")
    a.rows_per_batch = rows_per_batch
    return a


def kroquant_norm_residual(x: torch.Tensor, y: Optional[torch.Tensor] = None, *, gate: Optional[torch.Tensor] = None,
                           post_weight: Optional[torch.Tensor] = None, residual_scale: float = 1.0,
                           weight: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                           shift: Optional[torch.Tensor] = None, norm: str = "rms", post_norm: str = "none", eps: float = 1e-6,
                           rows_per_batch: Optional[int] = None, h_out: Optional[torch.Tensor] = None,
                           n_out: Optional[torch.Tensor] = None, branch_dtype: Optional[torch.dtype] = None, stream=None):
    """The step between two sub-blocks, one pass: -> (h, n) with

        h = residual_scale * x + gate * post_norm(y) * post_weight
        n = norm(h) * weight * (1 + scale) + shift

    x [rows, d] is the residual stream, y [rows, d] the branch (None: h = residual_scale * x, which is x itself for 1.0
    and is then not written unless h_out is given).  norm / post_norm: "none", "rms" or "layer".  gate, scale, shift:
    [d] or [batches, d] (row t uses row t // rows_per_batch); weight, post_weight: [d]; one dtype for all five.  x and h
    share a dtype, y and n share one (``branch_dtype`` without y): equal, or a float32 stream with a 16-bit branch.
    norm "none": n is None.  h_out may be x and n_out may be y."""
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    shape = x.shape
    a = _norm_args(shape[0], shape[1], norm, post_norm, residual_scale, eps, rows_per_batch, gate, post_weight, weight, scale, shift)
    a.ld_x = _rows2d(x, shape, "x")
    a.x, a.stream_dtype = x.data_ptr(), _DTYPES[x.dtype]
    if y is not None:
        a.ld_y = _rows2d(y, shape, "y")
        a.y, branch_dtype = y.data_ptr(), y.dtype
    elif branch_dtype is None:
        branch_dtype = x.dtype
    if branch_dtype not in _DTYPES:
        raise ValueError("branch_dtype must be float32, bfloat16 or float16")
    a.branch_dtype = _DTYPES[branch_dtype]
    h, n = h_out, n_out
    if h is not None:
        a.ld_h = _rows2d(h, shape, "h_out")
        if h.dtype is not x.dtype:
            raise ValueError("h_out must have x's dtype")
        a.h = h.data_ptr()
    elif y is not None or residual_scale != 1.0 or norm == "none":
        h = _empty_rows(x, x.dtype, stream)
        a.h, a.ld_h = h.data_ptr(), shape[1]
    if norm == "none":
        n = None
    elif n is not None:
        a.ld_n = _rows2d(n, shape, "n_out")
        if n.dtype is not branch_dtype:
            raise ValueError("n_out must have the branch's dtype")
        a.n = n.data_ptr()
    else:
        n = _empty_rows(x, branch_dtype, stream)
        a.n, a.ld_n = n.data_ptr(), shape[1]
    rc = load_library().kroquant_norm_residual(C.addressof(a), _stream(stream))
    if rc:
        raise KroQuantError(rc, "kroquant_norm_residual")
    return (x if h is None else h), n


def kroquant_norm_residual_grad(dn: Optional[torch.Tensor], h: torch.Tensor, *, dh: Optional[torch.Tensor] = None,
                                y: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                                post_weight: Optional[torch.Tensor] = None, residual_scale: float = 1.0,
                                weight: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                                shift: Optional[torch.Tensor] = None, norm: str = "rms", post_norm: str = "none",
                                eps: float = 1e-6, rows_per_batch: Optional[int] = None, stream=None) -> dict:
    """Backward pass of :func:`kroquant_norm_residual` (same vectors and settings): dn, dh = gradients at n and h (dh None:
    zero; dn None with norm "none"), h as the forward wrote it, y the branch.  -> dict with dx, with dy if y is given, and
    a float32 gradient ("dgate", "dpost_weight", "dweight", "dscale", "dshift") in the shape of every vector given."""
    if h.dim() != 2:
        raise ValueError("h must be [rows, d]")
    shape = h.shape
    rows, d = shape
    a = _norm_args(rows, d, norm, post_norm, residual_scale, eps, rows_per_batch, gate, post_weight, weight, scale, shift)
    a.ld_h = _rows2d(h, shape, "h")
    a.h, a.stream_dtype = h.data_ptr(), _DTYPES[h.dtype]
    if (dn is None) != (norm == "none"):
        raise ValueError("dn goes with a norm")
    branch_dtype = dn.dtype if dn is not None else y.dtype if y is not None else h.dtype
    if dn is not None:
        a.ld_dn = _rows2d(dn, shape, "dn")
        a.dn = dn.data_ptr()
    if dh is not None:
        a.ld_dh = _rows2d(dh, shape, "dh")
        if dh.dtype is not h.dtype:
            raise ValueError("dh must have h's dtype")
        a.dh = dh.data_ptr()
    if y is not None:
        a.ld_y = _rows2d(y, shape, "y")
        if y.dtype is not branch_dtype:
            raise ValueError("y and dn must share a dtype")
        a.y = y.data_ptr()
    elif gate is not None or post_weight is not None:
        raise ValueError("gate and post_weight act on the branch: y is needed")
    a.branch_dtype = _DTYPES[branch_dtype]
    with _allocating(stream):
        dx = _empty_rows(h, h.dtype, None)
        out = {"dx": dx}
        a.dx, a.ld_dx = dx.data_ptr(), d
        if y is not None:
            out["dy"] = dy = _empty_rows(h, branch_dtype, None)
            a.dy, a.ld_dy = dy.data_ptr(), d
        vectors = [(n, v.shape) for n, v in (("dgate", gate), ("dpost_weight", post_weight), ("dweight", weight), ("dscale", scale),
                                             ("dshift", shift)) if v is not None]
        if vectors:
            # the gradients are one allocation; the kernel's scratch space is another, so that it is free again after the call
            sizes = [s.numel() for _, s in vectors]
            a.dweight = 16                                                # any pointer: whether vector gradients are wanted at all
            nbytes = load_library().kroquant_norm_residual_grad_scratch_bytes(C.addressof(a))
            a.dweight = None
            store, scratch = h.new_empty(sum(sizes), dtype=torch.float32), h.new_empty(nbytes, dtype=torch.uint8)
            covered = (rows + a.rows_per_batch - 1) // a.rows_per_batch      # batches that have rows: the kernel writes those
            base, pos = store.data_ptr(), 0
            for (name, s), size in zip(vectors, sizes):
                out[name] = g = store.as_strided(s, (d, 1) if len(s) == 2 else (1,), pos)
                setattr(a, name, base + 4 * pos)
                if len(s) == 2 and s[0] > covered:
                    g.zero_()
                pos += size
            rc = load_library().kroquant_norm_residual_grad(C.addressof(a), scratch.data_ptr() if nbytes else None, nbytes, _stream(stream))
        else:
            rc = load_library().kroquant_norm_residual_grad(C.addressof(a), None, 0, _stream(stream))
    if rc:
        raise KroQuantError(rc, "kroquant_norm_residual_grad")
    return out


# ---- one step over new tokens: positions, the cache of keys and values, attention --------------------------------------
ROTARY_LAYOUTS = {"interleaved": 0, "half": 1}
CACHE_FORMATS = {"16bit": 0, "mxfp8": 1, "mxfp4": 2}


class _RotaryArgs(C.Structure):
    """kq_rotary_args_t (include/kroquant.h); arrays of two are two fields."""
    _fields_ = ([("dtype", C.c_int), ("batches", C.c_int64), ("tokens", C.c_int64)] +
                [(n, C.c_int) for n in ("head_dim", "layout", "inverse", "axes", "axis0", "axis1", "axis2", "axis3")] +
                [("frequencies", C.c_void_p), ("positions", C.c_void_p), ("positions_f32", C.c_int),
                 ("position_batch_stride", C.c_int64), ("position_token_stride", C.c_int64)] +
                [(n, C.c_void_p) for n in ("x0", "x1", "out0", "out1")] + [("heads0", C.c_int), ("heads1", C.c_int)] +
                [(n + i, C.c_int64) for n in ("x_batch_stride", "x_token_stride", "x_head_stride", "out_batch_stride", "out_token_stride",
                                              "out_head_stride") for i in "01"])


class _Cache(C.Structure):
    """kq_cache_t (include/kroquant.h)."""
    _fields_ = ([("format", C.c_int), ("dtype", C.c_int), ("pages", C.c_int64)] + [(n, C.c_int) for n in ("page_size", "heads", "head_dim")] +
                [(n, C.c_void_p) for n in ("k", "v", "k_scales", "v_scales")])


class _CacheRows(C.Structure):
    """kq_cache_rows_t (include/kroquant.h)."""
    _fields_ = [("rows", C.c_int64), ("sequences", C.c_int), ("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int),
                ("offsets", C.c_void_p), ("starts", C.c_void_p), ("dtype", C.c_int), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_row_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_row_stride", C.c_int64), ("v_head_stride", C.c_int64)]


class _AttentionArgs(C.Structure):
    """kq_attention_args_t (include/kroquant.h)."""
    _fields_ = ([(n, C.c_int) for n in ("sequences", "q_heads", "q_dtype", "out_dtype")] + [("q", C.c_void_p), ("out", C.c_void_p)] +
                [(n, C.c_int64) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride")] +
                [("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int), ("lengths", C.c_void_p), ("window", C.c_int),
                 ("scale", C.c_float), ("lse", C.c_void_p)])


# The same structs as bytes: packing one takes 1 us of a call, filling a ctypes structure 4.
_PACK_ROTARY = struct.Struct("@iqq8iPPiqq4P2i12q").pack
_PACK_ROWS = struct.Struct("@qiPqiPPiPPqqqq").pack
_PACK_ATTENTION = struct.Struct("@4iPPqqqqPqiPifP").pack


@functools.lru_cache(maxsize=256)
def _axes_of(axes, pairs: int, d: int):
    """Number of axes and their channels, filled up to four (a plan by sizes alone)."""
    axes = (2 * pairs,) if axes is None else axes
    if not 1 <= len(axes) <= 4 or any(a < 0 or a % 2 for a in axes) or sum(axes) != 2 * pairs or not 0 < 2 * pairs <= d:
        raise ValueError("axes: one to four even numbers of channels, together twice the frequencies and at most d")
    return len(axes), axes + (0, 0, 0)[: 4 - len(axes)]


def rotary_frequencies(axes, theta: float = 10000.0, device="cuda") -> torch.Tensor:
    """float64 [sum(axes) / 2]: theta ** (-2 i / a) for the a / 2 pairs of every axis of a channels."""
    return torch.cat([theta ** (-torch.arange(0, a, 2, dtype=torch.float64) / a) for a in axes]).to(device)


def _apart(t: torch.Tensor) -> bool:
    """Whether the elements of t lie at different addresses."""
    if t.is_contiguous():
        return True
    dims = list(zip(t.stride(), t.shape))
    for order in (dims[::-1], None):                                     # most often the last dimension is the innermost
        reach = 1
        for stride, size in order or sorted(dims):
            if size > 1:
                if stride < reach:
                    break
                reach += stride * (size - 1)
        else:
            return True
    return False


def _heads_last(t: torch.Tensor, what: str, dims: int, dtypes=_DTYPES) -> None:
    stride = t.stride()
    if len(stride) != dims or t.dtype not in dtypes or t.get_device() != _device() or (stride[-1] != 1 and t.shape[-1] > 1):
        raise ValueError(f"{what} must be a {dims}-D CUDA tensor of {', '.join(str(d)[6:] for d in dtypes)} on the current device with contiguous channels")


def _same_rows(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two tensors of one shape and dtype are the same elements in the same order."""
    return a is b or a.data_ptr() == b.data_ptr() and all(s == t for n, s, t in zip(a.shape, a.stride(), b.stride()) if n > 1)


def _turned_into(q: torch.Tensor, k: Optional[torch.Tensor], out, dims: int, others):
    """The outputs a caller gave :func:`kroquant_rotary`: each its input, or apart from all that the call reads and writes (others: besides q and k)."""
    outs = (out, None) if k is None else tuple(out)
    if len(outs) != 2 or not isinstance(outs[0], torch.Tensor) or (k is not None and not isinstance(outs[1], torch.Tensor)):
        raise ValueError("out must be a tensor, or a pair of tensors where k is given")
    ins = (q,) if k is None else (q, k)
    spans = [_span(x) for x in ins]
    rest = [(t, _span(t)) for t in others]
    seen = []                                                            # outputs, and the inputs that are none
    for x, o, span in zip(ins, outs, spans):
        if o is not x:
            _heads_last(o, "out", dims)
            if o.shape != x.shape or o.dtype is not q.dtype:
                raise ValueError("out must have its input's shape and dtype")
        if not _apart(o):
            raise ValueError("out must have elements of their own")
        if not _same_rows(o, x):
            place = _span(o)
            if _spans_meet(o, place, x, span):
                raise ValueError("out may be its input, but must not overlap it in another way")
            rest.append((x, span))
            span = place
        seen.append((o, span))
    # each output against the other one and against what is only read (its own input among that: once more)
    if len(seen) == 2 and _spans_meet(*seen[0], *seen[1]) or any(_spans_meet(*o, *t) for o in seen for t in rest):
        raise ValueError("out of q must overlap neither k nor out of k, out of k not q, and none the positions or frequencies")
    return outs


def kroquant_rotary(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, frequencies: torch.Tensor, *, axes=None,
                    layout: str = "interleaved", inverse: bool = False, out=None, stream=None):
    """Rotary positions: -> q turned, or (q, k) turned where k is given.

    q, k: [tokens, heads, d] or [batch, tokens, heads, d] of one dtype, each with its own number of heads, any strides with
    contiguous channels.  positions: int32 or float32 [tokens, axes] ([tokens] for one axis; [batch, tokens, axes] per sample).
    axes: channels of each axis (time, height, width, ...; up to four, each even), by default one axis of all the frequencies'
    pairs; frequencies: float64 [sum(axes) / 2] (:func:`rotary_frequencies`).  Pair p of axis i turns by
    positions[t, i] * frequencies[p], formed in 64 bits; channels behind the axes are copied.  layout: "interleaved" pairs
    (2p, 2p + 1) or "half" (p, p + pairs).  inverse turns back: the backward pass, with the gradients in place of q and k.
    out: tensor, or pair of tensors with k, to write to; each may be its input, and nothing else that the call touches."""
    shape, qt, dtype, dev = q.shape, q.stride(), q.dtype, _device()
    dims = len(shape)
    if dims not in (3, 4) or dtype not in _DTYPES or q.get_device() != dev or (qt[-1] != 1 and shape[-1] > 1):
        raise ValueError("q must be a CUDA float32, bfloat16 or float16 tensor [tokens, heads, d] or [batch, tokens, heads, d] on the current device "
                         "with contiguous channels")
    d, tokens, batches = shape[-1], shape[-3], shape[0] if dims == 4 else 1
    if k is not None:
        ks, kt = k.shape, k.stride()
        if len(ks) != dims or k.dtype is not dtype or k.get_device() != dev or ks[-1] != d or ks[-3] != tokens or (dims == 4 and ks[0] != batches) or \
                (kt[-1] != 1 and d > 1):
            raise ValueError("k must have q's dtype, device and shape but for the number of heads, and contiguous channels")
    pairs = frequencies.numel()
    if frequencies.dtype is not torch.float64 or frequencies.dim() != 1 or frequencies.get_device() != dev or not frequencies.is_contiguous():
        raise ValueError("frequencies must be a contiguous CUDA float64 tensor [pairs]")
    n, wide = _axes_of(None if axes is None else tuple(axes), pairs, d)
    way = ROTARY_LAYOUTS.get(layout)
    if way is None:
        raise ValueError(f"layout must be one of {sorted(ROTARY_LAYOUTS)}")
    place, ps = positions.shape, positions.stride()
    if n == 1 and len(place) == 1:
        place, ps = (place[0], 1), (ps[0], 1)
    if (positions.dtype is not torch.int32 and positions.dtype is not torch.float32) or positions.get_device() != dev or \
            (place != (tokens, n) and (dims != 4 or place != (batches, tokens, n))) or (n > 1 and ps[-1] != 1):
        raise ValueError("positions must be a CUDA int32 or float32 tensor [tokens, axes], or [batch, tokens, axes], with contiguous axes")
    no_k = k is None
    if out is None:
        qo, ko = _empty_rows(q, dtype, stream), None if no_k else _empty_rows(k, dtype, stream)
    else:
        qo, ko = _turned_into(q, k, out, dims, (positions, frequencies))
    ot = qo.stride()
    if no_k:
        kt = pt = (0, 0, 0, 0)
    else:
        pt = ko.stride()
    batched = dims == 4
    a = _PACK_ROTARY(_DTYPES[dtype], batches, tokens, d, way, 1 if inverse else 0, n, *wide, frequencies.data_ptr(),
                     positions.data_ptr(), 1 if positions.dtype is torch.float32 else 0, ps[0] if len(ps) == 3 else 0, ps[-2],
                     q.data_ptr(), 0 if no_k else k.data_ptr(), qo.data_ptr(), 0 if no_k else ko.data_ptr(), shape[-2], 0 if no_k else ks[-2],
                     qt[0] if batched else 0, kt[0] if batched else 0, qt[-3], kt[-3], qt[-2], kt[-2],
                     ot[0] if batched else 0, pt[0] if batched else 0, ot[-3], pt[-3], ot[-2], pt[-2])
    rc = load_library().kroquant_rotary(a, _stream(stream))
    if rc:
        raise KroQuantError(rc, "kroquant_rotary")
    return qo if no_k else (qo, ko)


class KVCache:
    """A paged cache of keys and values (kq_cache_t): `pages` pages of `page_size` positions for `heads` heads of head_dim channels,
    as they are ("16bit") or in MXFP8 or MXFP4.  The buffers are torch tensors: k, v [pages, heads, page_size, row] (16-bit values of
    `dtype`, or uint8 codes) and for the codes k_scales, v_scales uint8 [pages, heads, page_size, scale row]; a row has
    32 * ceil(head_dim / 32) channels, those behind head_dim zero.  dtype is what :func:`kroquant_cache_read` gives unless asked
    for another.  Which pages belong to which sequence is the caller's table.  Buffers that overlap (keys that are the values, too) can be
    read but not written."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scales: Optional[torch.Tensor] = None, v_scales: Optional[torch.Tensor] = None, *,
                 head_dim: int, format: str = "mxfp4", dtype=None):
        code = CACHE_FORMATS.get(format)
        if code is None:
            raise ValueError(f"format must be one of {sorted(CACHE_FORMATS)}")
        if not 1 <= head_dim <= 256:
            raise ValueError("head_dim must be in 1 .. 256")
        channels = 32 * ((head_dim + 31) // 32)
        row = channels if code < 2 else channels // 2
        if k.dim() != 4 or k.shape[-1] != row or v.shape != k.shape or v.dtype is not k.dtype or min(k.shape) < 1:
            raise ValueError(f"k and v must be [pages, heads, page_size, {row}]")
        if k.dtype is not torch.uint8 if code else k.dtype not in X_DTYPES:
            raise ValueError("k and v must be uint8 codes" if code else "k and v must be bfloat16 or float16")
        if code == 0:
            if dtype not in (None, k.dtype) or k_scales is not None or v_scales is not None:
                raise ValueError("a 16bit cache has its buffers' dtype and no scales")
            dtype = k.dtype
        else:
            dtype = torch.bfloat16 if dtype is None else dtype
            if dtype not in X_DTYPES:
                raise ValueError("dtype must be bfloat16 or float16")
            scales = tuple(k.shape[:3]) + (4 * ((channels + 127) // 128),)
            for t in (k_scales, v_scales):
                if t is None or t.dtype is not torch.uint8 or tuple(t.shape) != scales:
                    raise ValueError(f"k_scales and v_scales must be uint8 {list(scales)}")
        for t in (k, v) if code == 0 else (k, v, k_scales, v_scales):
            if not t.is_contiguous() or t.get_device() != k.get_device():
                raise ValueError("the cache's buffers must be contiguous tensors on one device")
        self._buffers = (k, v, k_scales, v_scales)
        own = [t for t in self._buffers if t is not None]
        self._shared = any(_meet(a, b) for i, a in enumerate(own) for b in own[:i])      # may be read, but not written
        self.format, self.dtype, self.head_dim, self.device = format, dtype, head_dim, k.device
        self.pages, self.heads, self.page_size = k.shape[0], k.shape[1], k.shape[2]
        self._device, self._c = k.get_device(), _Cache(code, _DTYPES[dtype], k.shape[0], k.shape[2], k.shape[1], head_dim, k.data_ptr(), v.data_ptr(),
                                                       None if code == 0 else k_scales.data_ptr(), None if code == 0 else v_scales.data_ptr())
        self._at = C.addressof(self._c)

    # (the C struct points into these: a cache keeps the buffers it was made with)
    k, v, k_scales, v_scales = (property(lambda self, i=i: self._buffers[i]) for i in range(4))

    @classmethod
    def empty(cls, pages: int, page_size: int, heads: int, head_dim: int, format: str = "mxfp4", dtype=torch.bfloat16, device="cuda") -> "KVCache":
        """A cache of zeros."""
        if format not in CACHE_FORMATS:
            raise ValueError(f"format must be one of {sorted(CACHE_FORMATS)}")
        channels, make = 32 * ((head_dim + 31) // 32), lambda row, dt: torch.zeros((pages, heads, page_size, row), dtype=dt, device=device)
        if format == "16bit":
            return cls(make(channels, dtype), make(channels, dtype), head_dim=head_dim, format=format)
        row, scales = channels if format == "mxfp8" else channels // 2, 4 * ((channels + 127) // 128)
        return cls(make(row, torch.uint8), make(row, torch.uint8), make(scales, torch.uint8), make(scales, torch.uint8), head_dim=head_dim,
                   format=format, dtype=dtype)


def _int_vector(t: torch.Tensor, size: int, dev: int, what: str) -> int:
    if t.dtype is not torch.int32 or t.shape != (size,) or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 tensor [{size}] on the cache's device")
    return t.data_ptr()


def _table(cache: KVCache, table: torch.Tensor):
    """(sequences, pointer, stride, width) of a table of pages, on the cache's device, which must be the current one."""
    dev, shape, stride = cache._device, table.shape, table.stride()
    if dev != _device():
        raise ValueError("the cache is not on the current CUDA device")
    if table.dtype is not torch.int32 or len(shape) != 2 or table.get_device() != dev or (shape[1] > 1 and stride[1] != 1) or \
            (shape[0] > 1 and stride[0] < 0):
        raise ValueError("table must be an int32 tensor [sequences, pages of a sequence] on the cache's device with contiguous rows")
    return shape[0], table.data_ptr(), stride[0], shape[1]


def _cache_rows(call: str, cache: KVCache, k, v, rows, where, offsets, starts, stream) -> None:
    n, table, stride, width = where
    (k_row, k_head, _), (v_row, v_head, _) = k.stride(), v.stride()
    a = _PACK_ROWS(rows, n, table, stride, width, 0 if offsets is None else _int_vector(offsets, n + 1, cache._device, "offsets"),
                   0 if starts is None else _int_vector(starts, n, cache._device, "starts"), _DTYPES[k.dtype], k.data_ptr(), v.data_ptr(),
                   k_row, k_head, v_row, v_head)
    rc = getattr(load_library(), call)(cache._at, a, _stream(stream))
    if rc:
        raise KroQuantError(rc, call)


def kroquant_cache_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, *, offsets: Optional[torch.Tensor] = None,
                         starts: Optional[torch.Tensor] = None, stream=None) -> None:
    """Keys and values of new tokens into the cache, encoded as it holds them.  k, v [rows, heads, head_dim] bfloat16 or float16 (a 16bit
    cache: its dtype), any strides with contiguous channels.  table int32 [sequences, n]: the pages of each sequence in order.
    offsets int32 [sequences + 1]: rows offsets[s] .. offsets[s + 1] - 1 belong to sequence s (None: one row per sequence); starts
    int32 [sequences]: the position of each sequence's first row (None: 0).  All three are read on the device; a row whose
    position lies before 0 or beyond the table, or whose table entry is no page (-1, say), is left out.  No place may be written twice by
    one call (a page that two sequences have, or one has twice)."""
    where = _table(cache, table)
    _heads_last(k, "k", 3, X_DTYPES)
    _heads_last(v, "v", 3, X_DTYPES)
    shape, dtype = k.shape, k.dtype
    rows = shape[0]
    if cache._shared:
        raise ValueError("the cache's buffers overlap: it can only be read")
    if shape != (rows, cache.heads, cache.head_dim) or v.shape != shape or v.dtype is not dtype or (cache.format == "16bit" and dtype is not cache.dtype):
        raise ValueError("k and v must be [rows, heads, head_dim] of the cache, of one dtype (a 16bit cache: its own)")
    if offsets is None and rows != where[0]:
        raise ValueError("without offsets there is one row per sequence")
    _cache_rows("kroquant_cache_write", cache, k, v, rows, where, offsets, starts, stream)


def kroquant_cache_read(cache: KVCache, table: torch.Tensor, rows: int, *, offsets: Optional[torch.Tensor] = None,
                        starts: Optional[torch.Tensor] = None, dtype=None, out=None, stream=None):
    """The inverse of :func:`kroquant_cache_write`: -> (k, v) [rows, heads, head_dim] in `dtype` (default: the cache's; float32 is allowed), the
    values that the cache holds at the places of the rows.  Rows without a place are zeros; rows outside the sequences
    (before offsets[0], from offsets[-1] on) are left as they are.  out: a pair of tensors to write to, which do not overlap (pages of a 16bit
    cache among them, where the call reads others: a copy of pages)."""
    where = _table(cache, table)
    shape = (rows, cache.heads, cache.head_dim)
    if out is None:
        dtype = cache.dtype if dtype is None else dtype
        if dtype not in _DTYPES:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        strides = (shape[1] * shape[2], shape[2], 1)
        if stream is None:
            k = torch.empty_strided(shape, strides, dtype=dtype, device=cache.device)                # (2.4 us by its shape alone)
            v = torch.empty_like(k)
        else:
            with _allocating(stream):
                k, v = (torch.empty_strided(shape, strides, dtype=dtype, device=cache.device) for _ in range(2))
    else:
        k, v = out
        for t in (k, v):
            _heads_last(t, "out", 3)
            if t.shape != shape or t.dtype is not k.dtype or dtype not in (None, t.dtype) or not _apart(t):
                raise ValueError("out must be two tensors [rows, heads, head_dim] of one dtype with elements of their own")
        if _meet(k, v):
            raise ValueError("the two tensors of out must not overlap")
    if offsets is None and rows != where[0]:
        raise ValueError("without offsets there is one row per sequence")
    _cache_rows("kroquant_cache_read", cache, k, v, rows, where, offsets, starts, stream)
    return k, v


def kroquant_cache_attention(q: torch.Tensor, cache: KVCache, table: torch.Tensor, lengths: torch.Tensor, *, scale: Optional[float] = None,
                             window: int = 0, out: Optional[torch.Tensor] = None, out_dtype=None, lse: bool = False, stream=None):
    """Attention of one new token of every sequence over its pages: -> out [sequences, q_heads, head_dim], softmax(scale q K^T) V
    over positions max(0, lengths - window) .. lengths - 1 (window 0: from 0); with lse also the float32 [sequences, q_heads]
    logarithms of the sums of exponentials.  q [sequences, q_heads, head_dim] bfloat16 or float16 (a 16bit cache: its dtype),
    q_heads a multiple of the cache's heads: query head h reads cache head h // (q_heads / heads).  scale: default
    head_dim ** -0.5.  lengths int32 [sequences] counts the new token, written before; it is read on the device.  A sequence
    without positions (length 0, no pages) gives zeros and -inf.  out_dtype: default q's.  out overlaps neither q nor the cache."""
    where = _table(cache, table)
    _heads_last(q, "q", 3, X_DTYPES)
    n, heads, d = q.shape
    if n != where[0] or d != cache.head_dim or heads < 1 or heads % cache.heads or (cache.format == "16bit" and q.dtype is not cache.dtype):
        raise ValueError("q must be [sequences, q_heads, head_dim], q_heads a multiple of the cache's heads (a 16bit cache: its dtype)")
    if window < 0:
        raise ValueError("window must not be negative")
    if out is None:
        out_dtype = q.dtype if out_dtype is None else out_dtype
        if out_dtype not in _DTYPES:
            raise ValueError("out_dtype must be float32, bfloat16 or float16")
        out = _empty_rows(q, out_dtype, stream)
    else:
        _heads_last(out, "out", 3)
        if out.shape != q.shape or out_dtype not in (None, out.dtype) or not _apart(out):
            raise ValueError("out must have q's shape and elements of its own")
        place = _span(out)
        if _spans_meet(out, place, q, _span(q)) or any(t is not None and _spans_meet(out, place, t, _span(t)) for t in cache._buffers):
            raise ValueError("out must overlap neither q nor the cache")
    lib, logs, scratch = load_library(), None, None
    if lse:
        with _allocating(stream):
            logs = torch.empty((n, heads), dtype=torch.float32, device=q.device)
    (q_row, q_head, _), (o_row, o_head, _) = q.stride(), out.stride()
    a = _PACK_ATTENTION(n, heads, _DTYPES[q.dtype], _DTYPES[out.dtype], q.data_ptr(), out.data_ptr(), q_row, q_head, o_row, o_head,
                        where[1], where[2], where[3], _int_vector(lengths, n, cache._device, "lengths"), min(window, 0x7FFFFFFF),
                        d ** -0.5 if scale is None else scale, 0 if logs is None else logs.data_ptr())
    nbytes = lib.kroquant_cache_attention_scratch_bytes(cache._at, a)
    if nbytes:
        if stream is None:
            scratch = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
        else:
            with _allocating(stream):
                scratch = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    rc = lib.kroquant_cache_attention(cache._at, a, None if scratch is None else scratch.data_ptr(), nbytes, _stream(stream))
    if rc:
        raise KroQuantError(rc, "kroquant_cache_attention")
    return (out, logs) if lse else out


_GEMM_PAIR = True


def set_gemm_pair(on: bool) -> None:
    """Which GEMM variant THIS BINDING passes with its calls from now on (a default of the Python layer, handed to
    the library per call or per calibration handle; the library keeps no process-wide switch): pairs of CTAs on
    256 x 256 tiles (default) or one CTA per tile."""
    global _GEMM_PAIR
    _GEMM_PAIR = bool(on)


class Calibrator:
    """Handle of a kroquant_calib_t: layer-wise calibration of the transform (Section 3.3).

    A [M, d] and W [o, d] are contiguous CUDA bfloat16 tensors; they are kept alive by this object.
    """

    def __init__(self, A: torch.Tensor, W: torch.Tensor, n_sets: int = 1, stream=None):
        for t in (A, W):
            if t.dim() != 2 or t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("A and W must be contiguous 2-D CUDA bfloat16 tensors")
        if A.shape[1] != W.shape[1]:
            raise ValueError("A [M, d] and W [o, d] must share d")
        self.A, self.W, self.n_sets = A, W, n_sets
        self.M, self.d, self.o = A.shape[0], A.shape[1], W.shape[0]
        out = C.c_void_p()
        _check(load_library().kroquant_calib_create(_ptr(A), _ptr(W), self.M, self.o, self.d, n_sets,
                                                    _stream(stream), C.byref(out)), "kroquant_calib_create")
        self._h = out

    def destroy(self) -> None:
        if getattr(self, "_h", None):
            load_library().kroquant_calib_destroy(self._h)
            self._h = None

    __del__ = destroy

    def _get(self, name: str, shape) -> np.ndarray:
        out = np.empty(shape, np.float32)
        _check(getattr(load_library(), "kroquant_calib_get_" + name)(self._h, out.ctypes.data_as(C.c_void_p)),
               "kroquant_calib_get_" + name)
        return out

    @property
    def theta(self) -> np.ndarray:
        return self._get("theta", (self.n_sets, 5, 3))

    @theta.setter
    def theta(self, value) -> None:
        v = np.ascontiguousarray(value, dtype=np.float32)
        if v.shape != (self.n_sets, 5, 3):
            raise ValueError("theta must have shape [n_sets, 5, 3]")
        _check(load_library().kroquant_calib_set_theta(self._h, v.ctypes.data_as(C.c_void_p)), "kroquant_calib_set_theta")

    @property
    def lambdas(self) -> np.ndarray:
        return self._get("lambdas", (2,))

    @lambdas.setter
    def lambdas(self, value) -> None:
        v = np.ascontiguousarray(value, dtype=np.float32)
        if v.shape != (2,):
            raise ValueError("lambdas = (lambda_A, lambda_W)")
        _check(load_library().kroquant_calib_set_lambdas(self._h, v.ctypes.data_as(C.c_void_p)),
               "kroquant_calib_set_lambdas")

    def factors(self) -> np.ndarray:
        """G [n_sets, 5, 2, 2] of the current parameters (input of Factors.create)."""
        return self._get("factors", (self.n_sets, 5, 2, 2))

    def weight_factors(self) -> np.ndarray:
        """H [n_sets, 5, 2, 2] with H_k = G_k^-T: the Kronecker set of T^-T, for quantizing W offline."""
        return self._get("weight_factors", (self.n_sets, 5, 2, 2))

    def loss_grad(self, grad: bool = True, stream=None):
        """-> (losses float64 [3] = (L_out, L_A, L_W), dL/dtheta float32 [n_sets, 5, 3] or None)."""
        losses = np.empty(3, np.float64)
        g = np.empty((self.n_sets, 5, 3), np.float32) if grad else None
        _check(load_library().kroquant_calib_set_gemm_variant(self._h, int(_GEMM_PAIR)), "kroquant_calib_set_gemm_variant")
        _check(load_library().kroquant_calib_loss_grad(self._h, losses.ctypes.data_as(C.c_void_p),
                                                       g.ctypes.data_as(C.c_void_p) if grad else None,
                                                       _stream(stream)), "kroquant_calib_loss_grad")
        return losses, g

    def run(self, steps: int, lr: float = 1e-2, history: bool = True, stream=None):
        """`steps` Adam steps; -> history float64 [steps + 1, 3] (or None, asynchronous)."""
        h = np.empty((steps + 1, 3), np.float64) if history else None
        _check(load_library().kroquant_calib_set_gemm_variant(self._h, int(_GEMM_PAIR)), "kroquant_calib_set_gemm_variant")
        _check(load_library().kroquant_calib_run(self._h, steps, lr, h.ctypes.data_as(C.c_void_p) if history else None,
                                                 _stream(stream)), "kroquant_calib_run")
        return h
