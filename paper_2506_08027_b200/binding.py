"""Thin ctypes binding of libmxfp8.so: argument marshalling only.

Every function has the name and argument order of its C entry point in ``include/mxfp8.h``
and takes torch tensors (device memory) where C takes device pointers.  Nothing here
computes: a missing library or a non-zero status raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

FP32, BF16 = 0, 1
ROW, COL, BOTH = 1, 2, 3
RULE_PAPER, RULE_OCP = 0, 1
E4M3, E5M2 = 0, 1
E2M3, E3M2, E2M1 = 3, 4, 5          # MXFP6 / MXFP4 elements: conversion kernels only
SF_LINEAR, SF_SWIZZLED = 0, 1
K_MAJOR, MN_MAJOR = 0, 1
ERR_NULL, ERR_ENUM, ERR_SHAPE, ERR_ALIGN, ERR_UNSUPPORTED, ERR_CUDA = -1, -2, -3, -4, -5, -6
ERR_DEVICE_TIMEOUT, ERR_WORKSPACE, ERR_DEVICE_ARGS = -7, -8, -9
ACT_NONE, ACT_RELU, ACT_RELU2, ACT_SILU, ACT_GELU_TANH = 0, 1, 2, 3, 4

EXPORTS = (
    "mxfp8_quantize", "mxfp8_dequantize", "mxfp8_gemm", "mxfp8_scale_bytes", "mxfp8_sf_offset",
    "mxfp8_gemm_workspace_bytes", "mxfp8_device_status", "mxfp8_status_string",
    "mxfp8_launch_count", "mxfp8_quantize_host_ws_bytes", "mxfp8_quantize_host",
    "mxfp8_linear_host_ws_bytes", "mxfp8_linear_host", "mxfp8_fake_quantize", "mxfp8_linear_ws_bytes",
    "mxfp8_linear", "mxfp8_grouped_gemm", "mxfp8_quantize_multi", "mxfp8_gemm_multi", "mxfp8_act_quantize", "mxfp8_rmsnorm_quantize",
    "mxfp8_rmsnorm_quantize_static", "mxfp8_rmsnorm_quantize_static_max_rows", "mxfp8_glu_quantize",
    "mxfp8_sf_concat_k", "mxfp8_gemm_reduce_scatter", "mxfp8_enable_peer_access", "mxfp8_gemm_last_clock", "mxfp8_layernorm_quantize", "mxfp8_act_grad_quantize",
    "mxfp8_moe_rows", "mxfp8_moe_sort_ws_bytes", "mxfp8_moe_sort", "mxfp8_moe_dispatch_quantize", "mxfp8_moe_combine", "mxfp8_moe_combine_grad",
    "mxfp8_e2m1_packed_bytes", "mxfp8_e2m1_pack", "mxfp8_e2m1_matvec", "mxfp8_e2m1_moe_ws_bytes", "mxfp8_e2m1_moe",
    "mxfp8_residual_rmsnorm", "mxfp8_residual_rmsnorm_quantize", "mxfp8_residual_rmsnorm_grad_ws_bytes", "mxfp8_residual_rmsnorm_grad",
    "mxfp8_grad_ws_bytes", "mxfp8_grad_sumsq", "mxfp8_grad_scale", "mxfp8_grad_clip",
)


class Mxfp8Error(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__("%s failed: %d (%s)" % (what, status, status_string(status)))
        self.status = status


class _QuantizeItem(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("q_row", ctypes.c_void_p), ("s_row", ctypes.c_void_p),
                ("q_col", ctypes.c_void_p), ("s_col", ctypes.c_void_p)]


class _GemmProblem(ctypes.Structure):
    _fields_ = [("Aq", ctypes.c_void_p), ("As", ctypes.c_void_p), ("Bq", ctypes.c_void_p), ("Bs", ctypes.c_void_p),
                ("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("a_major", ctypes.c_int), ("b_major", ctypes.c_int), ("a_elem", ctypes.c_int), ("b_elem", ctypes.c_int),
                ("D", ctypes.c_void_p)]


class _Seam(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("block_dtype", ctypes.c_int), ("stream_dtype", ctypes.c_int), ("param_dtype", ctypes.c_int),
                ("gamma_post", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("rows_per_gate", ctypes.c_int64), ("gamma_pre", ctypes.c_void_p),
                ("branch_scale", ctypes.c_float), ("residual_scale", ctypes.c_float), ("eps", ctypes.c_float)]


class _GradItem(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("numel", ctypes.c_int64), ("dtype", ctypes.c_int)]


class _Epilogue(ctypes.Structure):
    _fields_ = [("orientation", ctypes.c_int), ("scale_rule", ctypes.c_int), ("elem", ctypes.c_int),
                ("q_row", ctypes.c_void_p), ("s_row", ctypes.c_void_p),
                ("q_col", ctypes.c_void_p), ("s_col", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load (building first if the sources are newer) the CUDA library; fail loudly."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if os.environ.get("MXFP8_NO_BUILD") != "1":
            path = _build.build()
        if not os.path.exists(path):
            raise ImportError("libmxfp8.so is missing: run `python -m paper_2506_08027_b200.build`")
        _lib = load_library(path)
    return _lib


def load_library(path: str) -> ctypes.CDLL:
    """dlopen a build of the library and declare every entry point's signature."""
    L = ctypes.CDLL(path)
    i, i64, p, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    L.mxfp8_quantize.restype = i
    L.mxfp8_quantize.argtypes = [p, i, i64, i64, i, i, i, p, p, p, p, i, p]
    L.mxfp8_dequantize.restype = i
    L.mxfp8_dequantize.argtypes = [p, p, i64, i64, i, i, i, p, i, p]
    L.mxfp8_gemm.restype = i
    L.mxfp8_gemm.argtypes = [p, p, p, p, i64, i64, i64, i, i, i, i, p, i, ctypes.POINTER(_Epilogue), p, sz, p]
    L.mxfp8_scale_bytes.restype = sz
    L.mxfp8_scale_bytes.argtypes = [i64, i64, i, i]
    L.mxfp8_sf_offset.restype = i64
    L.mxfp8_sf_offset.argtypes = [i64, i64, i64, i]
    L.mxfp8_gemm_workspace_bytes.restype = sz
    L.mxfp8_gemm_workspace_bytes.argtypes = [i64, i64, i64, i, i]
    L.mxfp8_device_status.restype = i
    L.mxfp8_device_status.argtypes = [p]
    L.mxfp8_status_string.restype = ctypes.c_char_p
    L.mxfp8_status_string.argtypes = [i]
    L.mxfp8_launch_count.restype = i64
    L.mxfp8_launch_count.argtypes = []
    L.mxfp8_quantize_host_ws_bytes.restype = sz
    L.mxfp8_quantize_host_ws_bytes.argtypes = [i, i64, i64, i]
    L.mxfp8_quantize_host.restype = i
    L.mxfp8_quantize_host.argtypes = [p, i, i64, i64, i, i, i, p, p, p, p, i, p, sz, p]
    L.mxfp8_fake_quantize.restype = i
    L.mxfp8_fake_quantize.argtypes = [p, i, i64, i64, i, i, i, p, p, p]
    L.mxfp8_rmsnorm_quantize.restype = i
    L.mxfp8_rmsnorm_quantize.argtypes = [p, i, i64, i64, p, ctypes.c_float, p, i, i, i, p, p, p, p, i, p]
    L.mxfp8_layernorm_quantize.restype = i
    L.mxfp8_layernorm_quantize.argtypes = [p, i, i64, i64, p, p, ctypes.c_float, p, p, i, i, i, p, p, p, p, i, p]
    L.mxfp8_rmsnorm_quantize_static.restype = i
    L.mxfp8_rmsnorm_quantize_static.argtypes = [p, i, i64, i64, p, ctypes.c_float, i, i, i, p, p, p, p, i, p]
    L.mxfp8_rmsnorm_quantize_static_max_rows.restype = i64
    L.mxfp8_rmsnorm_quantize_static_max_rows.argtypes = []
    L.mxfp8_glu_quantize.restype = i
    L.mxfp8_glu_quantize.argtypes = [p, i, i64, i64, i, i, i, i, p, p, p, p, i, p]
    L.mxfp8_act_grad_quantize.restype = i
    L.mxfp8_act_grad_quantize.argtypes = [p, p, i, i64, i64, i, i, i, i, p, p, p, p, i, p]
    L.mxfp8_act_quantize.restype = i
    L.mxfp8_act_quantize.argtypes = [p, i, i64, i64, i, i, i, i, p, p, p, p, i, p]
    L.mxfp8_gemm_multi.restype = i
    L.mxfp8_gemm_multi.argtypes = [ctypes.POINTER(_GemmProblem), i, i, p]
    L.mxfp8_quantize_multi.restype = i
    L.mxfp8_quantize_multi.argtypes = [ctypes.POINTER(_QuantizeItem), i, i, i, i, i, i, p]
    L.mxfp8_grouped_gemm.restype = i
    L.mxfp8_grouped_gemm.argtypes = [p, p, p, p, p, i, i, i64, i64, i64, i, i, i, p, i, p]
    L.mxfp8_moe_rows.restype = i64
    L.mxfp8_moe_rows.argtypes = [i64, i, i]
    L.mxfp8_moe_sort_ws_bytes.restype = sz
    L.mxfp8_moe_sort_ws_bytes.argtypes = [i64, i, i]
    L.mxfp8_moe_sort.restype = i
    L.mxfp8_moe_sort.argtypes = [p, i64, i, i, p, p, p, i64, p, sz, p]
    L.mxfp8_moe_dispatch_quantize.restype = i
    L.mxfp8_moe_dispatch_quantize.argtypes = [p, i, i64, i64, p, i64, i, p, p, i, i, i, i, p, p, p, p, i, p]
    L.mxfp8_moe_combine.restype = i
    L.mxfp8_moe_combine.argtypes = [p, i, i64, i64, p, p, i64, i, p, i, p]
    L.mxfp8_moe_combine_grad.restype = i
    L.mxfp8_moe_combine_grad.argtypes = [p, i, i64, i64, p, i, i64, p, p, i, p, p, i, p, p, p]
    L.mxfp8_e2m1_packed_bytes.restype = sz
    L.mxfp8_e2m1_packed_bytes.argtypes = [i64, i64, i64]
    L.mxfp8_e2m1_pack.restype = i
    L.mxfp8_e2m1_pack.argtypes = [p, p, i64, i64, i64, p, p]
    L.mxfp8_e2m1_matvec.restype = i
    L.mxfp8_e2m1_matvec.argtypes = [p, i64, i64, p, i64, i64, p, i, p, i, p]
    L.mxfp8_e2m1_moe_ws_bytes.restype = sz
    L.mxfp8_e2m1_moe_ws_bytes.argtypes = [i64, i, i64]
    L.mxfp8_e2m1_moe.restype = i
    L.mxfp8_e2m1_moe.argtypes = [p, p, i64, i64, i, i, p, p, i64, i, i, p, i, p, p, p, sz, p]
    seam = ctypes.POINTER(_Seam)
    L.mxfp8_residual_rmsnorm.restype = i
    L.mxfp8_residual_rmsnorm.argtypes = [seam, p, p, p, p, p, p, p]
    L.mxfp8_residual_rmsnorm_quantize.restype = i
    L.mxfp8_residual_rmsnorm_quantize.argtypes = [seam, p, p, p, p, p, i, i, i, p, p, p, p, i, p]
    L.mxfp8_residual_rmsnorm_grad_ws_bytes.restype = sz
    L.mxfp8_residual_rmsnorm_grad_ws_bytes.argtypes = [seam]
    L.mxfp8_residual_rmsnorm_grad.restype = i
    L.mxfp8_residual_rmsnorm_grad.argtypes = [seam, p, p, p, p, p, p, p, p, p, p, p, p, sz, p]
    items = ctypes.POINTER(_GradItem)
    L.mxfp8_grad_ws_bytes.restype = sz
    L.mxfp8_grad_ws_bytes.argtypes = [items, i]
    L.mxfp8_grad_sumsq.restype = i
    L.mxfp8_grad_sumsq.argtypes = [items, i, p, p, sz, p]
    L.mxfp8_grad_scale.restype = i
    L.mxfp8_grad_scale.argtypes = [items, i, p, ctypes.c_float, p, p]
    L.mxfp8_grad_clip.restype = i
    L.mxfp8_grad_clip.argtypes = [items, i, ctypes.c_float, p, p, sz, p]
    L.mxfp8_gemm_last_clock.restype = i
    L.mxfp8_gemm_last_clock.argtypes = [p, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    L.mxfp8_enable_peer_access.restype = i
    L.mxfp8_enable_peer_access.argtypes = [i]
    L.mxfp8_sf_concat_k.restype = i
    L.mxfp8_sf_concat_k.argtypes = [p, i, i64, i64, p, p]
    L.mxfp8_gemm_reduce_scatter.restype = i
    L.mxfp8_gemm_reduce_scatter.argtypes = [p, p, p, p, i64, i64, i64, i, i, i, i, ctypes.POINTER(ctypes.c_void_p), i, i, p]
    L.mxfp8_linear_ws_bytes.restype = sz
    L.mxfp8_linear_ws_bytes.argtypes = [i64, i64, i64]
    L.mxfp8_linear.restype = i
    L.mxfp8_linear.argtypes = [p, p, p, i64, i64, i64, i, p, p, p, p, sz, p]
    L.mxfp8_linear_host_ws_bytes.restype = sz
    L.mxfp8_linear_host_ws_bytes.argtypes = [i64, i64, i64]
    L.mxfp8_linear_host.restype = i
    L.mxfp8_linear_host.argtypes = [p, p, p, i64, i64, i64, i, p, p, p, p, sz, p]
    return L


def status_string(status: int) -> str:
    return lib().mxfp8_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != 0:
        raise Mxfp8Error(status, what)


def _ptr(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("the C entry points take dense row-major buffers: pass a contiguous tensor")
    return t.data_ptr()           # the declared argument types turn it into a pointer (0, an empty tensor's, into NULL)


# torch.cuda.current_stream() builds a Stream object (3 us of the 10 to 12 us that a call through this module took); the
# handle alone costs a tenth of a microsecond.  Every torch that this library builds against has it; the public call
# stands in if one day it does not.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream=None):
    if stream is None and _raw_stream is not None:
        return _raw_stream(_current_device())
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return FP32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("source must be float32 or bfloat16")


def mxfp8_scale_bytes(rows: int, cols: int, orientation: int, sf_layout: int) -> int:
    return int(lib().mxfp8_scale_bytes(rows, cols, orientation, sf_layout))


def mxfp8_sf_offset(mn: int, kblock: int, n_kblocks: int, sf_layout: int) -> int:
    return int(lib().mxfp8_sf_offset(mn, kblock, n_kblocks, sf_layout))


def mxfp8_gemm_workspace_bytes(M: int, N: int, K: int, out_dtype: int, has_epilogue: bool) -> int:
    return int(lib().mxfp8_gemm_workspace_bytes(M, N, K, out_dtype, int(has_epilogue)))


def mxfp8_device_status(stream=None) -> int:
    return int(lib().mxfp8_device_status(_stream(stream)))


def mxfp8_launch_count() -> int:
    return int(lib().mxfp8_launch_count())


def alloc_quantize_outputs(rows: int, cols: int, orientation: int, sf_layout: int, device="cuda"):
    """Caller-side allocation helper: (q_row, s_row, q_col, s_col), None where unused."""
    out = []
    for o in (ROW, COL):
        if orientation & o:
            out.append(torch.empty((rows, cols), dtype=torch.uint8, device=device))
            out.append(torch.empty(mxfp8_scale_bytes(rows, cols, o, sf_layout), dtype=torch.uint8, device=device))
        else:
            out += [None, None]
    return tuple(out)


def mxfp8_quantize(src: torch.Tensor, orientation: int, scale_rule: int, elem: int,
                   q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    rows, cols = src.shape
    assert src.is_contiguous()
    _check(lib().mxfp8_quantize(_ptr(src), _dtype_code(src), rows, cols, orientation, scale_rule, elem,
                                _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout,
                                _stream(stream)), "mxfp8_quantize")


def mxfp8_dequantize(q: torch.Tensor, s: torch.Tensor, orientation: int, elem: int, sf_layout: int,
                     dst: torch.Tensor, stream=None) -> None:
    rows, cols = q.shape
    _check(lib().mxfp8_dequantize(_ptr(q), _ptr(s), rows, cols, orientation, elem, sf_layout,
                                  _ptr(dst), _dtype_code(dst), _stream(stream)), "mxfp8_dequantize")


def make_epilogue(orientation: int, scale_rule: int, elem: int, q_row=None, s_row=None, q_col=None, s_col=None):
    e = _Epilogue()
    e.orientation, e.scale_rule, e.elem = orientation, scale_rule, elem
    e.q_row = None if q_row is None else q_row.data_ptr()
    e.s_row = None if s_row is None else s_row.data_ptr()
    e.q_col = None if q_col is None else q_col.data_ptr()
    e.s_col = None if s_col is None else s_col.data_ptr()
    e._keep = (q_row, s_row, q_col, s_col)
    return e


def mxfp8_gemm(Aq, As, Bq, Bs, M: int, N: int, K: int, a_major: int, b_major: int, a_elem: int,
               b_elem: int, D, epi=None, workspace=None, stream=None) -> None:
    out_dtype = FP32 if D is None else _dtype_code(D)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().mxfp8_gemm(_ptr(Aq), _ptr(As), _ptr(Bq), _ptr(Bs), M, N, K, a_major, b_major,
                            a_elem, b_elem, _ptr(D), out_dtype,
                            None if epi is None else ctypes.byref(epi),
                            _ptr(workspace), ws_bytes, _stream(stream)), "mxfp8_gemm")


def mxfp8_quantize_host_ws_bytes(src_dtype: int, rows: int, cols: int, orientation: int) -> int:
    return int(lib().mxfp8_quantize_host_ws_bytes(src_dtype, rows, cols, orientation))


def mxfp8_quantize_host(src_host: torch.Tensor, orientation: int, scale_rule: int, elem: int,
                        q_row_host, s_row_host, q_col_host, s_col_host, sf_layout: int,
                        dev_ws: torch.Tensor, stream=None) -> None:
    rows, cols = src_host.shape
    _check(lib().mxfp8_quantize_host(_ptr(src_host), _dtype_code(src_host), rows, cols, orientation,
                                     scale_rule, elem, _ptr(q_row_host), _ptr(s_row_host),
                                     _ptr(q_col_host), _ptr(s_col_host), sf_layout, _ptr(dev_ws),
                                     dev_ws.numel() * dev_ws.element_size(), _stream(stream)),
           "mxfp8_quantize_host")


def mxfp8_linear_host_ws_bytes(T: int, H: int, F: int) -> int:
    return int(lib().mxfp8_linear_host_ws_bytes(T, H, F))


def mxfp8_linear_host(x_host, w_host, dy_host, scale_rule: int, y_host, dx_host, dw_host,
                      dev_ws: torch.Tensor, stream=None) -> None:
    T, H = x_host.shape
    F = w_host.shape[0]
    _check(lib().mxfp8_linear_host(_ptr(x_host), _ptr(w_host), _ptr(dy_host), T, H, F, scale_rule,
                                   _ptr(y_host), _ptr(dx_host), _ptr(dw_host), _ptr(dev_ws),
                                   dev_ws.numel() * dev_ws.element_size(), _stream(stream)),
           "mxfp8_linear_host")


def mxfp8_fake_quantize(src: torch.Tensor, orientation: int, scale_rule: int, elem: int,
                        dst_row, dst_col, stream=None) -> None:
    rows, cols = src.shape
    _check(lib().mxfp8_fake_quantize(_ptr(src), _dtype_code(src), rows, cols, orientation, scale_rule, elem,
                                     _ptr(dst_row), _ptr(dst_col), _stream(stream)), "mxfp8_fake_quantize")


def mxfp8_linear_ws_bytes(T: int, H: int, F: int) -> int:
    return int(lib().mxfp8_linear_ws_bytes(T, H, F))


def mxfp8_linear(x, w, dy, scale_rule: int, y, dx, dw, ws, stream=None) -> None:
    T, H = x.shape
    F = w.shape[0]
    _check(lib().mxfp8_linear(_ptr(x), _ptr(w), _ptr(dy), T, H, F, scale_rule, _ptr(y), _ptr(dx), _ptr(dw),
                              _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "mxfp8_linear")


GROUP_M, GROUP_K = 1, 2


def mxfp8_grouped_gemm(aq, a_s, bq, b_s, group_offsets: torch.Tensor, mode: int, M: int, N: int, K: int,
                       b_major: int, a_elem: int, b_elem: int, D: torch.Tensor, stream=None) -> None:
    assert group_offsets.dtype == torch.int32 and group_offsets.is_cuda
    _check(lib().mxfp8_grouped_gemm(_ptr(aq), _ptr(a_s), _ptr(bq), _ptr(b_s), _ptr(group_offsets),
                                    group_offsets.numel() - 1, mode, M, N, K, b_major, a_elem, b_elem,
                                    _ptr(D), _dtype_code(D), _stream(stream)), "mxfp8_grouped_gemm")


def mxfp8_sf_concat_k(parts: torch.Tensor, num_parts: int, mn: int, k_part: int, dst: torch.Tensor, stream=None) -> None:
    _check(lib().mxfp8_sf_concat_k(_ptr(parts), num_parts, mn, k_part, _ptr(dst), _stream(stream)), "mxfp8_sf_concat_k")


def mxfp8_gemm_last_clock(stream=None):
    """(SM MHz, microseconds) of the most recent GEMM launch, measured by the kernel itself; waits for the stream."""
    mhz, us = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib().mxfp8_gemm_last_clock(_stream(stream), ctypes.byref(mhz), ctypes.byref(us)), "mxfp8_gemm_last_clock")
    return mhz.value, us.value


def mxfp8_enable_peer_access(peer_device: int) -> None:
    _check(lib().mxfp8_enable_peer_access(peer_device), "mxfp8_enable_peer_access")


def make_owner_pointers(addresses):
    """addresses: one device address per owner (int, or a tensor whose data_ptr() is taken).  Returns the
    host pointer array mxfp8_gemm_reduce_scatter takes; build it once per set of buffers."""
    arr = (ctypes.c_void_p * len(addresses))()
    for k, a in enumerate(addresses):
        arr[k] = a.data_ptr() if isinstance(a, torch.Tensor) else int(a)
    return arr


def mxfp8_gemm_reduce_scatter(aq, a_s, bq, b_s, M: int, N: int, K: int, a_major: int, b_major: int, a_elem: int, b_elem: int,
                              owners, first_owner: int, stream=None) -> None:
    _check(lib().mxfp8_gemm_reduce_scatter(_ptr(aq), _ptr(a_s), _ptr(bq), _ptr(b_s), M, N, K, a_major, b_major, a_elem, b_elem,
                                           owners, len(owners), first_owner, _stream(stream)), "mxfp8_gemm_reduce_scatter")


def make_quantize_items(entries):
    """entries: sequence of (src, q_row, s_row, q_col, s_col) tensors (None where unused).  Returns the
    ctypes array mxfp8_quantize_multi takes; build it once and reuse it while the tensors live."""
    arr = (_QuantizeItem * len(entries))()
    for k, (src, q_row, s_row, q_col, s_col) in enumerate(entries):
        assert src.is_contiguous()
        arr[k].src = src.data_ptr()
        arr[k].rows, arr[k].cols = src.shape
        arr[k].q_row, arr[k].s_row, arr[k].q_col, arr[k].s_col = _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col)
    return arr


def mxfp8_quantize_multi(items, src_dtype: int, orientation: int, scale_rule: int, elem: int, sf_layout: int,
                         stream=None) -> None:
    _check(lib().mxfp8_quantize_multi(items, len(items), src_dtype, orientation, scale_rule, elem, sf_layout,
                                      _stream(stream)), "mxfp8_quantize_multi")


def make_gemm_problems(entries):
    """entries: sequence of (Aq, As, Bq, Bs, M, N, K, a_major, b_major, a_elem, b_elem, D).  Returns the ctypes
    array mxfp8_gemm_multi takes; build it once and reuse it while the tensors live."""
    arr = (_GemmProblem * len(entries))()
    for k, (aq, a_s, bq, b_s, M, N, K, a_major, b_major, a_elem, b_elem, D) in enumerate(entries):
        arr[k].Aq, arr[k].As, arr[k].Bq, arr[k].Bs = aq.data_ptr(), a_s.data_ptr(), bq.data_ptr(), b_s.data_ptr()
        arr[k].M, arr[k].N, arr[k].K = M, N, K
        arr[k].a_major, arr[k].b_major, arr[k].a_elem, arr[k].b_elem = a_major, b_major, a_elem, b_elem
        arr[k].D = D.data_ptr()
    return arr


def mxfp8_gemm_multi(problems, out_dtype: int, stream=None) -> None:
    _check(lib().mxfp8_gemm_multi(problems, len(problems), out_dtype, _stream(stream)), "mxfp8_gemm_multi")


def mxfp8_act_grad_quantize(dh: torch.Tensor, z: torch.Tensor, act: int, orientation: int, scale_rule: int, elem: int,
                            q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    rows, cols = z.shape
    assert z.is_contiguous() and dh.is_contiguous() and dh.shape == z.shape and dh.dtype == z.dtype
    _check(lib().mxfp8_act_grad_quantize(_ptr(dh), _ptr(z), _dtype_code(z), rows, cols, act, orientation, scale_rule, elem,
                                         _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout,
                                         _stream(stream)), "mxfp8_act_grad_quantize")


def mxfp8_act_quantize(src: torch.Tensor, act: int, orientation: int, scale_rule: int, elem: int,
                       q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    rows, cols = src.shape
    assert src.is_contiguous()
    _check(lib().mxfp8_act_quantize(_ptr(src), _dtype_code(src), rows, cols, act, orientation, scale_rule, elem,
                                    _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout,
                                    _stream(stream)), "mxfp8_act_quantize")


def mxfp8_layernorm_quantize(src: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, eps: float, mean: torch.Tensor, rstd: torch.Tensor,
                             orientation: int, scale_rule: int, elem: int,
                             q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    rows, cols = src.shape
    assert src.is_contiguous() and gamma.dtype == src.dtype and beta.dtype == src.dtype
    assert mean.dtype == torch.float32 and rstd.dtype == torch.float32
    _check(lib().mxfp8_layernorm_quantize(_ptr(src), _dtype_code(src), rows, cols, _ptr(gamma), _ptr(beta), eps, _ptr(mean), _ptr(rstd),
                                          orientation, scale_rule, elem, _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout,
                                          _stream(stream)), "mxfp8_layernorm_quantize")


def mxfp8_rmsnorm_quantize(src: torch.Tensor, gamma: torch.Tensor, eps: float, rstd: torch.Tensor,
                           orientation: int, scale_rule: int, elem: int,
                           q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    rows, cols = src.shape
    assert src.is_contiguous() and gamma.dtype == src.dtype and gamma.numel() == cols
    assert rstd.dtype == torch.float32 and rstd.numel() == rows
    _check(lib().mxfp8_rmsnorm_quantize(_ptr(src), _dtype_code(src), rows, cols, _ptr(gamma), eps, _ptr(rstd),
                                        orientation, scale_rule, elem, _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col),
                                        sf_layout, _stream(stream)), "mxfp8_rmsnorm_quantize")


def mxfp8_rmsnorm_quantize_static_max_rows() -> int:
    return int(lib().mxfp8_rmsnorm_quantize_static_max_rows())


def mxfp8_rmsnorm_quantize_static(src: torch.Tensor, gamma: torch.Tensor, eps: float,
                                  orientation: int, scale_rule: int, elem: int,
                                  q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    rows, cols = src.shape
    assert src.is_contiguous() and gamma.dtype == src.dtype and gamma.numel() == cols
    _check(lib().mxfp8_rmsnorm_quantize_static(_ptr(src), _dtype_code(src), rows, cols, _ptr(gamma), eps,
                                               orientation, scale_rule, elem, _ptr(q_row), _ptr(s_row), _ptr(q_col),
                                               _ptr(s_col), sf_layout, _stream(stream)), "mxfp8_rmsnorm_quantize_static")


def mxfp8_glu_quantize(src: torch.Tensor, act: int, orientation: int, scale_rule: int, elem: int,
                       q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    """src: [rows, 2 * cols] = (gate | up); the outputs have shape [rows, cols]."""
    rows, two_cols = src.shape
    assert src.is_contiguous() and two_cols % 2 == 0
    _check(lib().mxfp8_glu_quantize(_ptr(src), _dtype_code(src), rows, two_cols // 2, act, orientation, scale_rule, elem,
                                    _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout,
                                    _stream(stream)), "mxfp8_glu_quantize")


def _addresses(*tensors):
    """Addresses of a call's tensors (None for one that is left out), looked at once: they are dense and lie on the current device."""
    device = _current_device()
    out = []
    for t in tensors:
        if t is None:
            out.append(None)
        elif t.get_device() != device:                           # -1 for a host tensor
            raise ValueError("a tensor of shape %s is on %s, the call runs on cuda:%d" % (tuple(t.shape), t.device, device))
        elif not t.is_contiguous():
            raise ValueError("the C entry points take dense row-major buffers: pass a contiguous tensor")
        else:
            out.append(t.data_ptr())
    return out


def _stream_for(stream, *tensors) -> int:
    """The call's stream, after a look at its tensors: all of them lie on the device that the stream belongs to and that
    is current (a launch elsewhere would read foreign addresses)."""
    device = _current_device()
    if stream is not None and stream.device.index != device:
        raise ValueError("the call runs on the current device, cuda:%d: its stream belongs to %s" % (device, stream.device))
    for t in tensors:
        if t is not None and t.get_device() != device:           # -1 for a host tensor
            raise ValueError("a tensor of shape %s is on %s, the call runs on cuda:%d" % (tuple(t.shape), t.device, device))
    return _stream(stream)


def _int32(*tensors) -> None:
    for t in tensors:
        if t is not None and t.dtype is not torch.int32:
            raise TypeError("indexes and offsets must be int32")


def mxfp8_moe_rows(tokens: int, top_k: int, num_experts: int) -> int:
    return int(lib().mxfp8_moe_rows(tokens, top_k, num_experts))


def mxfp8_moe_sort_ws_bytes(tokens: int, top_k: int, num_experts: int) -> int:
    return int(lib().mxfp8_moe_sort_ws_bytes(tokens, top_k, num_experts))


def mxfp8_moe_sort(expert_ids: torch.Tensor, num_experts: int, group_offsets: torch.Tensor, row_of: torch.Tensor, slot_of: torch.Tensor,
                   ws=None, stream=None) -> None:
    """expert_ids, row_of: [tokens, top_k]; group_offsets: [num_experts + 1]; slot_of: [rows], rows >= mxfp8_moe_rows(...)."""
    tokens, top_k = expert_ids.shape
    _int32(expert_ids, group_offsets, row_of, slot_of)
    st = _stream_for(stream, expert_ids, group_offsets, row_of, slot_of, ws)
    if group_offsets.numel() != num_experts + 1 or row_of.shape != expert_ids.shape:
        raise ValueError("group_offsets holds num_experts + 1 numbers, row_of has the shape of expert_ids")
    _check(lib().mxfp8_moe_sort(_ptr(expert_ids), tokens, top_k, num_experts, _ptr(group_offsets), _ptr(row_of), _ptr(slot_of), slot_of.numel(),
                                _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), st), "mxfp8_moe_sort")


def mxfp8_moe_dispatch_quantize(src: torch.Tensor, slot_of: torch.Tensor, top_k: int, weights, group_offsets: torch.Tensor,
                                orientation: int, scale_rule: int, elem: int, q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    """src: [tokens, cols]; slot_of: [rows]; weights: None or FP32 [tokens, top_k]; outputs as mxfp8_quantize of [rows, cols]."""
    tokens, cols = src.shape
    rows = slot_of.numel()
    _int32(slot_of, group_offsets)
    st = _stream_for(stream, src, slot_of, weights, group_offsets, q_row, s_row, q_col, s_col)
    _float_weights(weights, tokens, top_k)
    if orientation & ROW and q_row is not None and s_row is not None:
        _holds(q_row, s_row, rows, cols, rows, cols // 32, sf_layout)
    if orientation & COL and q_col is not None and s_col is not None:
        _holds(q_col, s_col, rows, cols, cols, rows // 32, sf_layout)
    _check(lib().mxfp8_moe_dispatch_quantize(_ptr(src), _dtype_code(src), tokens, cols, _ptr(slot_of), rows, top_k, _ptr(weights),
                                             _ptr(group_offsets), group_offsets.numel() - 1, orientation, scale_rule, elem,
                                             _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout, st),
           "mxfp8_moe_dispatch_quantize")


def _holds(q, s, rows: int, cols: int, mn: int, blocks: int, sf_layout: int) -> None:
    """Codes and scales of a [rows, cols] conversion with `mn` x `blocks` scales fit their buffers."""
    need = mn * blocks if sf_layout == SF_LINEAR else (mn + 127) // 128 * ((blocks + 3) // 4) * 512
    if q.nbytes < rows * cols or s.nbytes < need:
        raise ValueError("an output is smaller than [%d, %d] needs" % (rows, cols))


def _float_weights(weights, tokens: int, top_k: int) -> None:
    if weights is not None and (weights.dtype is not torch.float32 or weights.shape != (tokens, top_k)):
        raise TypeError("weights must be float32 [tokens, top_k]")


def mxfp8_moe_combine(src: torch.Tensor, row_of: torch.Tensor, weights, dst: torch.Tensor, stream=None) -> None:
    """src: [rows, cols]; row_of: [tokens, top_k]; weights: None or FP32 [tokens, top_k]; dst: [tokens, cols]."""
    rows, cols = src.shape
    tokens, top_k = row_of.shape
    _int32(row_of)
    st = _stream_for(stream, src, row_of, weights, dst)
    _float_weights(weights, tokens, top_k)
    if dst.shape != (tokens, cols):
        raise ValueError("dst must be [tokens, cols]")
    _check(lib().mxfp8_moe_combine(_ptr(src), _dtype_code(src), rows, cols, _ptr(row_of), _ptr(weights), tokens, top_k, _ptr(dst),
                                   _dtype_code(dst), st), "mxfp8_moe_combine")


def mxfp8_moe_combine_grad(dy: torch.Tensor, src, row_of: torch.Tensor, slot_of, weights, group_offsets, d_src, d_weights, stream=None) -> None:
    """dy: [tokens, cols]; src, d_src: [rows, cols]; row_of, weights, d_weights: [tokens, top_k]; d_src or d_weights may be None.  Without d_weights
    src may be None, without d_src slot_of and group_offsets may."""
    tokens, cols = dy.shape
    sorted_rows = src if src is not None else d_src
    if sorted_rows is None:
        raise ValueError("src or d_src is needed")
    rows = sorted_rows.shape[0]
    _int32(row_of, slot_of, group_offsets)
    st = _stream_for(stream, dy, src, row_of, slot_of, weights, group_offsets, d_src, d_weights)
    top_k = row_of.shape[1]
    _float_weights(weights, tokens, top_k)
    _float_weights(d_weights, tokens, top_k)
    if row_of.shape[0] != tokens or sorted_rows.shape[1] != cols or (slot_of is not None and slot_of.numel() != rows) or \
            (d_src is not None and (d_src.shape != sorted_rows.shape or d_src.dtype != sorted_rows.dtype)):
        raise ValueError("shapes or types of dy, src, d_src, row_of and slot_of do not agree")
    num_groups = 1 if group_offsets is None else group_offsets.numel() - 1
    _check(lib().mxfp8_moe_combine_grad(_ptr(dy), _dtype_code(dy), tokens, cols, _ptr(src), _dtype_code(sorted_rows), rows, _ptr(row_of), _ptr(slot_of), top_k,
                                        _ptr(weights), _ptr(group_offsets), num_groups, _ptr(d_src), _ptr(d_weights), st),
           "mxfp8_moe_combine_grad")


def mxfp8_e2m1_packed_bytes(num_matrices: int, rows: int, cols: int) -> int:
    return int(lib().mxfp8_e2m1_packed_bytes(num_matrices, rows, cols))


def mxfp8_e2m1_pack(q: torch.Tensor, s: torch.Tensor, num_matrices: int, packed: torch.Tensor, stream=None) -> None:
    """q: [num_matrices * rows, cols] E2M1 slots and s: their linear ROW scales, as mxfp8_quantize writes them."""
    all_rows, cols = q.shape
    st = _stream_for(stream, q, s, packed)
    if q.element_size() != 1 or s.element_size() != 1:
        raise TypeError("codes and scales are bytes")
    if num_matrices < 1 or all_rows % num_matrices:
        raise ValueError("q holds num_matrices matrices of the same number of rows")
    rows = all_rows // num_matrices
    if s.numel() * s.element_size() < all_rows * (cols // 32) or packed.numel() * packed.element_size() < mxfp8_e2m1_packed_bytes(num_matrices, rows, cols):
        raise ValueError("s or packed is too small")
    _check(lib().mxfp8_e2m1_pack(_ptr(q), _ptr(s), num_matrices, rows, cols, _ptr(packed), st), "mxfp8_e2m1_pack")


def mxfp8_e2m1_matvec(x: torch.Tensor, packed: torch.Tensor, num_matrices: int, matrix_ids, y: torch.Tensor, stream=None) -> None:
    """x: BF16 [tokens, cols]; matrix_ids: None (one matrix) or int32 [tokens, choices]; y: [tokens * choices, rows]."""
    tokens, cols = x.shape
    if x.dtype != torch.bfloat16:
        raise TypeError("x must be bfloat16")
    _int32(matrix_ids)
    st = _stream_for(stream, x, packed, matrix_ids, y)
    per_token = 1 if matrix_ids is None else matrix_ids.shape[1]
    if (matrix_ids is not None and matrix_ids.shape[0] != tokens) or y.shape[0] != tokens * per_token:
        raise ValueError("y holds one row per token and choice")
    rows = y.shape[1]
    if packed.numel() * packed.element_size() < mxfp8_e2m1_packed_bytes(num_matrices, rows, cols):
        raise ValueError("packed is smaller than num_matrices matrices of [%d, %d]" % (rows, cols))
    _check(lib().mxfp8_e2m1_matvec(_ptr(x), tokens, cols, _ptr(packed), num_matrices, rows, _ptr(matrix_ids), per_token, _ptr(y),
                                   _dtype_code(y), st), "mxfp8_e2m1_matvec")


def mxfp8_e2m1_moe_ws_bytes(tokens: int, top_k: int, inner: int) -> int:
    return int(lib().mxfp8_e2m1_moe_ws_bytes(tokens, top_k, inner))


def _nbytes(t) -> int:
    return 0 if t is None else t.nbytes


def mxfp8_e2m1_moe(x: torch.Tensor, logits: torch.Tensor, top_k: int, gate_up: torch.Tensor, down: torch.Tensor, inner: int, act: int, renormalize: bool,
                   y: torch.Tensor, ids, weights, ws: torch.Tensor, stream=None) -> None:
    """x: BF16 [tokens, cols]; logits: FP32 [tokens, experts]; gate_up, down: packed [experts, 2 * inner, cols] and [experts, cols, inner];
    y: [tokens, cols]; ids, weights: None or int32 / FP32 [tokens, top_k]; ws: mxfp8_e2m1_moe_ws_bytes(...) bytes."""
    tokens, cols = x.shape
    experts = logits.shape[1]
    if x.dtype is not torch.bfloat16 or logits.dtype is not torch.float32:
        raise TypeError("x must be bfloat16 and logits float32")
    _int32(ids)
    st = _stream_for(stream)
    x_at, logits_at, gate_up_at, down_at, y_at, ids_at, weights_at, ws_at = _addresses(x, logits, gate_up, down, y, ids, weights, ws)
    _float_weights(weights, tokens, top_k)
    if logits.shape[0] != tokens or y.shape != x.shape or (ids is not None and ids.shape != (tokens, top_k)):
        raise ValueError("logits, y and ids hold one row per token")
    # tiles of 16 rows x 128 columns, 1088 bytes each (mxfp8_e2m1_packed_bytes)
    if _nbytes(gate_up) < experts * (-(-2 * inner // 16)) * (-(-cols // 128)) * 1088 or _nbytes(down) < experts * (-(-cols // 16)) * (-(-inner // 128)) * 1088:
        raise ValueError("gate_up or down is smaller than %d matrices of [%d, %d] and [%d, %d]" % (experts, 2 * inner, cols, cols, inner))
    _check(lib().mxfp8_e2m1_moe(x_at, logits_at, tokens, cols, experts, top_k, gate_up_at, down_at, inner, act, renormalize, y_at,
                                _dtype_code(y), ids_at, weights_at, ws_at, _nbytes(ws), st), "mxfp8_e2m1_moe")


class Seam:
    """The parameters of a seam between two blocks (see make_seam); holds its tensors as long as it lives."""

    __slots__ = ("gamma_pre", "gamma_post", "gate", "rows_per_gate", "c")

    def describe(self, rows: int, cols: int, block: int, stream: int) -> "_Seam":
        """The C description for tensors of this shape and types; a copy of its own, so that threads may share the seam."""
        if cols != self.gamma_pre.numel():
            raise ValueError("the seam's weights have %d columns, the tensors %d" % (self.gamma_pre.numel(), cols))
        if self.gate is not None and self.gate.shape[0] != -(-rows // self.rows_per_gate):
            raise ValueError("the gate has %d rows, %d rows of %d need %d" % (self.gate.shape[0], rows, self.rows_per_gate, -(-rows // self.rows_per_gate)))
        c = _Seam.from_buffer_copy(self.c)
        c.rows, c.cols, c.block_dtype, c.stream_dtype = rows, cols, block, stream
        return c


def make_seam(gamma_pre: torch.Tensor, gamma_post=None, gate=None, rows_per_gate: int = 1, branch_scale: float = 1.0, residual_scale: float = 1.0,
              eps: float = 1e-5) -> Seam:
    """gamma_pre, gamma_post (or None): [cols]; gate (or None): [ceil(rows / rows_per_gate), cols]; all of one type.  Their addresses are taken here."""
    given = [t for t in (gamma_pre, gamma_post, gate) if t is not None]
    if any(t.dtype is not gamma_pre.dtype or t.shape[-1] != gamma_pre.numel() for t in given) or gamma_pre.dim() != 1 or \
            (gamma_post is not None and gamma_post.dim() != 1) or (gate is not None and (gate.dim() != 2 or rows_per_gate < 1)):
        raise ValueError("gamma_pre and gamma_post are [cols], gate is [rows of the gate, cols], all of one type")
    s = Seam()
    s.gamma_pre, s.gamma_post, s.gate, s.rows_per_gate = gamma_pre, gamma_post, gate, int(rows_per_gate)
    s.c = _Seam(param_dtype=_dtype_code(gamma_pre), gamma_post=_ptr(gamma_post), gate=_ptr(gate), rows_per_gate=rows_per_gate, gamma_pre=_ptr(gamma_pre),
                branch_scale=branch_scale, residual_scale=residual_scale, eps=eps)
    return s


def _row_statistics(rows: int, *tensors) -> None:
    for t in tensors:
        if t is not None and (t.dtype is not torch.float32 or t.numel() != rows):
            raise TypeError("row statistics are float32 [rows]")


def _alike(what: str, shape, dtype, *tensors) -> None:
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.shape != shape):
            raise ValueError("%s have one shape and type" % what)


def mxfp8_residual_rmsnorm(seam: Seam, y: torch.Tensor, h_in: torch.Tensor, h: torch.Tensor, x, rstd_post, rstd_pre: torch.Tensor, stream=None) -> None:
    """y, x (or None): [rows, cols] of the block's type; h_in, h: of the stream's; rstd_post (or None), rstd_pre: FP32 [rows]."""
    rows, cols = shape = y.shape
    st = _stream_for(stream, seam.gamma_pre, seam.gamma_post, seam.gate)
    at = _addresses(y, h_in, h, x, rstd_post, rstd_pre)
    if x is not None:
        _alike("y and x", shape, y.dtype, x)
    _alike("y, h_in and h", shape, h_in.dtype, h_in, h)
    _row_statistics(rows, rstd_post, rstd_pre)
    c = seam.describe(rows, cols, _dtype_code(y), _dtype_code(h_in))
    _check(lib().mxfp8_residual_rmsnorm(c, *at, st), "mxfp8_residual_rmsnorm")


def mxfp8_residual_rmsnorm_quantize(seam: Seam, y: torch.Tensor, h_in: torch.Tensor, h: torch.Tensor, rstd_post, rstd_pre: torch.Tensor,
                                    orientation: int, scale_rule: int, elem: int, q_row, s_row, q_col, s_col, sf_layout: int, stream=None) -> None:
    """As mxfp8_residual_rmsnorm, with the next block's input converted: outputs as mxfp8_quantize of [rows, cols]."""
    rows, cols = y.shape
    st = _stream_for(stream, y, h_in, h, rstd_post, rstd_pre, seam.gamma_pre, seam.gamma_post, seam.gate, q_row, s_row, q_col, s_col)
    _alike("y, h_in and h", y.shape, h_in.dtype, h_in, h)
    _row_statistics(rows, rstd_post, rstd_pre)
    if orientation & ROW and q_row is not None and s_row is not None:
        _holds(q_row, s_row, rows, cols, rows, cols // 32, sf_layout)
    if orientation & COL and q_col is not None and s_col is not None:
        _holds(q_col, s_col, rows, cols, cols, rows // 32, sf_layout)
    c = seam.describe(rows, cols, _dtype_code(y), _dtype_code(h_in))
    _check(lib().mxfp8_residual_rmsnorm_quantize(c, _ptr(y), _ptr(h_in), _ptr(h), _ptr(rstd_post), _ptr(rstd_pre), orientation, scale_rule, elem,
                                                 _ptr(q_row), _ptr(s_row), _ptr(q_col), _ptr(s_col), sf_layout, st), "mxfp8_residual_rmsnorm_quantize")


def mxfp8_residual_rmsnorm_grad_ws_bytes(seam: Seam, rows: int, cols: int) -> int:
    """Bytes for any types of the tensors, on the current device."""
    return int(lib().mxfp8_residual_rmsnorm_grad_ws_bytes(seam.describe(rows, cols, FP32, FP32)))


def mxfp8_residual_rmsnorm_grad(seam: Seam, dx, dh, y: torch.Tensor, h: torch.Tensor, rstd_post, rstd_pre: torch.Tensor, dy, dh_in,
                                d_gamma_pre, d_gamma_post, d_gate, ws: torch.Tensor, stream=None) -> None:
    """dx, y, dy: [rows, cols] of the block's type; dh, h, dh_in: of the stream's; the weights' gradients: FP32 of their shapes.  dx, dh and
    every output may be None."""
    rows, cols = y.shape
    st = _stream_for(stream, dx, dh, y, h, rstd_post, rstd_pre, dy, dh_in, d_gamma_pre, d_gamma_post, d_gate, ws, seam.gamma_pre, seam.gamma_post, seam.gate)
    _alike("dx, y and dy", y.shape, y.dtype, dx, dy)
    _alike("y, dh, h and dh_in", y.shape, h.dtype, dh, h, dh_in)
    _row_statistics(rows, rstd_post, rstd_pre)
    for t, like in ((d_gamma_pre, seam.gamma_pre), (d_gamma_post, seam.gamma_post), (d_gate, seam.gate)):
        if t is not None and (like is None or t.dtype is not torch.float32 or t.shape != like.shape):
            raise ValueError("gradients of the seam's weights are float32 of the weights' shapes")
    c = seam.describe(rows, cols, _dtype_code(y), _dtype_code(h))
    _check(lib().mxfp8_residual_rmsnorm_grad(c, _ptr(dx), _ptr(dh), _ptr(y), _ptr(h), _ptr(rstd_post), _ptr(rstd_pre), _ptr(dy), _ptr(dh_in),
                                             _ptr(d_gamma_pre), _ptr(d_gamma_post), _ptr(d_gate), _ptr(ws), _nbytes(ws), st),
           "mxfp8_residual_rmsnorm_grad")


class GradItems:
    """The C table of a set of gradients (see make_grad_items); holds the tensors as long as it lives."""

    __slots__ = ("c", "count", "keep", "device")


def make_grad_items(grads, results=None) -> GradItems:
    """grads: FP32 / BF16 tensors of one device; results: where the scaled values go (None: in place).  Build it once and reuse it while the
    tensors keep their storage: it takes 2 to 3 us of host time per tensor, more than clipping many short ones does.  mxfp8_grad_sumsq needs no
    results.  What is written may overlap no other gradient (the same one twice, say)."""
    grads, results = list(grads), None if results is None else list(results)
    if results is not None and (len(results) != len(grads) or any(r.dtype is not g.dtype or r.shape != g.shape for g, r in zip(grads, results))):
        raise ValueError("results have the gradients' shapes and types")
    items = GradItems()
    items.c, items.count, items.keep = (_GradItem * max(1, len(grads)))(), len(grads), (grads, results)
    items.device = None
    for k, g in enumerate(grads):
        to = g if results is None else results[k]
        for t in (g, to):
            if not t.is_cuda or items.device not in (None, t.get_device()):
                raise ValueError("gradients lie on one CUDA device")
            items.device = t.get_device()
        items.c[k].src, items.c[k].dst, items.c[k].numel, items.c[k].dtype = _ptr(g), _ptr(to), g.numel(), _dtype_code(g)
    # what is written overlaps nothing else, else a value would be scaled twice or read after it was
    spans = sorted((c.dst, c.dst + t.nbytes, True, k) for k, (c, t) in enumerate(zip(items.c, grads)) if t.numel()) + \
        sorted((c.src, c.src + t.nbytes, False, k) for k, (c, t) in enumerate(zip(items.c, grads)) if t.numel() and c.src != c.dst)
    end, written_end = -1, -1                                # of all spans so far, of those that are written
    for lo, hi, written, _ in sorted(spans):
        if lo < (end if written else written_end):
            raise ValueError("a gradient that is written overlaps another one")
        end, written_end = max(end, hi), max(written_end, hi if written else -1)
    return items


def _grad_stream(stream, items: GradItems, *tensors) -> int:
    st = _stream_for(stream, *tensors)
    if items.device is not None and items.device != _current_device():
        raise ValueError("the gradients are on cuda:%d, the call runs on cuda:%d" % (items.device, _current_device()))
    return st


def mxfp8_grad_ws_bytes(items: GradItems) -> int:
    return int(lib().mxfp8_grad_ws_bytes(items.c, items.count))


def mxfp8_grad_sumsq(items: GradItems, sumsq: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """sumsq: one float64 on the device."""
    st = _grad_stream(stream, items, sumsq, ws)
    if sumsq.dtype is not torch.float64 or sumsq.numel() != 1:
        raise TypeError("sumsq is one float64")
    _check(lib().mxfp8_grad_sumsq(items.c, items.count, _ptr(sumsq), _ptr(ws), _nbytes(ws), st), "mxfp8_grad_sumsq")


def _norm_and_factor(norm: torch.Tensor) -> None:
    if norm.dtype is not torch.float32 or norm.numel() != 2:
        raise TypeError("norm is two float32: the norm and the factor")


def mxfp8_grad_scale(items: GradItems, sumsq: torch.Tensor, max_norm: float, norm: torch.Tensor, stream=None) -> None:
    """sumsq: one float64; norm: two float32, the norm and the factor."""
    st = _grad_stream(stream, items, sumsq, norm)
    if sumsq.dtype is not torch.float64 or sumsq.numel() != 1:
        raise TypeError("sumsq is one float64")
    _norm_and_factor(norm)
    _check(lib().mxfp8_grad_scale(items.c, items.count, _ptr(sumsq), max_norm, _ptr(norm), st), "mxfp8_grad_scale")


def mxfp8_grad_clip(items: GradItems, max_norm: float, norm: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """norm: two float32, the norm and the factor."""
    st = _grad_stream(stream, items, norm, ws)
    _norm_and_factor(norm)
    _check(lib().mxfp8_grad_clip(items.c, items.count, max_norm, _ptr(norm), _ptr(ws), _nbytes(ws), st), "mxfp8_grad_clip")
