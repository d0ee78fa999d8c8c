"""Thin ctypes binding of the root-mean-square normalization of libmtfm_hta.so (C ABI declared in include/mtfm_rms.h):
h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, in the element type or in 8 bits with a scale per row.
Argument checks and marshalling only; PyTorch supplies device memory and the stream.  There is no fallback: without the
built library the first call raises."""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

import torch

from . import hta

EXPORTS = ("mtfm_rms_fwd", "mtfm_rms_fwd_q8", "mtfm_rms_bwd", "mtfm_rms_bwd_workspace_bytes")
KERNEL_FWD, KERNEL_BWD, KERNEL_BWD_REDUCE = 7, 8, 9
KINDS = {torch.int8: 0, torch.float8_e4m3fn: 1}

_declared = None

# argument block of mtfm_binding_rms (struct RmsArgs of csrc/binding.hip), see hta.call_packed
_BLOCK = struct.Struct("10P5qif4i")
_FWD, _FWD_Q8, _BWD = 0, 1, 2


def load_library() -> ctypes.CDLL:
    global _declared
    if _declared is not None:
        return _declared
    lib = hta.load_library()
    vp, i32, i64, f32, sz, ci = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t,
                                 ctypes.c_int)
    lib.mtfm_rms_fwd.restype = ci
    lib.mtfm_rms_fwd.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, i32, f32, ci, vp]
    lib.mtfm_rms_fwd_q8.restype = ci
    lib.mtfm_rms_fwd_q8.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, i32, f32, ci, ci, vp]
    lib.mtfm_rms_bwd_workspace_bytes.restype = sz
    lib.mtfm_rms_bwd_workspace_bytes.argtypes = [i32]
    lib.mtfm_rms_bwd.restype = ci
    lib.mtfm_rms_bwd.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, i64, i32, ci, vp, sz, vp]
    lib.mtfm_binding_rms.restype = ci
    lib.mtfm_binding_rms.argtypes = [vp, vp]
    _declared = lib
    return lib


def _call(fields) -> None:
    status = (_declared or load_library()).mtfm_binding_rms(_BLOCK.pack(*fields, 0), hta._current_stream())
    if status != hta.OK:
        raise hta.HtaError(status, hta.mtfm_hta_last_error())


_workspace_words = {}  # of a backward call, by width (host arithmetic that never changes)
_CODES = {torch.bfloat16: hta.BF16, torch.float32: hta.FP32}


def _operand(x: torch.Tensor):
    """(shape, element type, its code) of the operand that the others are like."""
    if x.dim() != 2:
        raise ValueError(f"[rows, width] expected, got {tuple(x.shape)}")
    code = _CODES.get(x.dtype)
    if code is None:
        raise TypeError(f"unsupported element type {x.dtype}")
    return x.shape, x.dtype, code


def _rows(name: str, t: torch.Tensor, shape, dtype) -> int:
    """Row stride of an operand [rows, width] whose rows are contiguous."""
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name}: {tuple(shape)} {dtype} expected, got {tuple(t.shape)} {t.dtype}")
    if t.is_contiguous():
        return shape[1]
    if t.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    return t.stride(0)


def _vector(name: str, t: torch.Tensor, n: int) -> None:
    if t.dtype is not torch.float32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous float32 values expected, got {tuple(t.shape)} {t.dtype}")


def _out(name: str, t: torch.Tensor, shape, dtype) -> torch.Tensor:
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous {tuple(shape)} {dtype} expected, got {tuple(t.shape)} {t.dtype}")
    return t


def mtfm_rms_bwd_workspace_bytes(width: int) -> int:
    return int(load_library().mtfm_rms_bwd_workspace_bytes(width))


def _forward(call, x, weight, eps, residual, h, y, rstd, scale, kind, operand):
    shape, dtype, code = operand
    n, d = shape
    x_stride, r_stride = _rows("x", x, shape, dtype), 0
    _vector("weight", weight, d)
    P = hta._address
    if residual is not None:
        r_stride = _rows("residual", residual, shape, dtype)
        h = torch.empty_like(x, memory_format=torch.contiguous_format) if h is None else _out("h", h, shape, dtype)
    elif h is not None:
        raise ValueError("h without a residual is x")
    hta.check_on_current_device(x, weight, residual, h, y, rstd, scale)
    _call((x.data_ptr(), P(residual), weight.data_ptr(), P(h), y.data_ptr(), P(rstd), P(scale), 0, 0, 0, x_stride, r_stride, 0, n, 0,
           d, eps, code, kind, call))
    return x if h is None else h


def mtfm_rms_fwd(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                 y: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None, save_rstd: bool = True,
                 rstd: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(y, h, rstd) of rows x [n, width] (bf16 or float32) and weight [width] (float32).  h is the sum with the residual (x itself
    without one) and with rstd what the backward pass reads; rstd is None when save_rstd is False.  Outputs may be given, and may
    be the inputs' own memory (y is x, h is residual)."""
    operand = _operand(x)
    shape, dtype, _ = operand
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if y is None else _out("y", y, shape, dtype)
    if rstd is not None:
        _vector("rstd", rstd, shape[0])
    elif save_rstd:
        rstd = weight.new_empty(shape[0])
    return y, _forward(_FWD, x, weight, eps, residual, h, y, rstd, None, 0, operand), rstd


def mtfm_rms_fwd_q8(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                    kind: torch.dtype = torch.int8, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                    h: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(q, scale, h) with y = q * scale[:, None] in 8 bits, `kind` torch.int8 or torch.float8_e4m3fn."""
    if kind not in KINDS:
        raise TypeError(f"unsupported 8-bit type {kind}")
    operand = _operand(x)
    shape = operand[0]
    q = torch.empty_like(x, dtype=kind, memory_format=torch.contiguous_format) if q is None else _out("q", q, shape, kind)
    if scale is None:
        scale = weight.new_empty(shape[0])
    _vector("scale", scale, shape[0])
    return q, scale, _forward(_FWD_Q8, x, weight, eps, residual, h, q, None, scale, KINDS[kind], operand)


def mtfm_rms_bwd(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, dh: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dx, dweight) for the gradients dy of y and dh of h; dx is the gradient of x and of the residual.  `out` may hold preallocated
    (dx, dweight); dx may be dy or dh."""
    shape, dtype, code = _operand(h)
    n, d = shape
    h_stride, dy_stride = _rows("h", h, shape, dtype), _rows("dy", dy, shape, dtype)
    dh_stride = 0 if dh is None else _rows("dh", dh, shape, dtype)
    _vector("weight", weight, d)
    _vector("rstd", rstd, n)
    dx, dweight = out or (None, None)
    dx = torch.empty_like(h, memory_format=torch.contiguous_format) if dx is None else _out("dx", dx, shape, dtype)
    if dweight is None:
        dweight = torch.empty_like(weight)
    _vector("dweight", dweight, d)
    if workspace is None:
        words = _workspace_words.get(d)
        if words is None:
            words = _workspace_words[d] = max(mtfm_rms_bwd_workspace_bytes(d), 256) // 4
        workspace = weight.new_empty(words)
    elif not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    hta.check_on_current_device(dy, h, weight, rstd, dh, dx, dweight, workspace)
    P = hta._address
    _call((h.data_ptr(), P(dh), weight.data_ptr(), 0, dx.data_ptr(), rstd.data_ptr(), 0, dy.data_ptr(), dweight.data_ptr(),
           workspace.data_ptr(), h_stride, dh_stride, dy_stride, n, workspace.numel() * workspace.element_size(), d, 0.0, code, 0, _BWD))
    return dx, dweight
