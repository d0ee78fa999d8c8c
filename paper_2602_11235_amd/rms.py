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


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return hta.BF16
    if t.dtype == torch.float32:
        return hta.FP32
    raise TypeError(f"unsupported element type {t.dtype}")


def _rows(name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None) -> int:
    """Row stride of an operand [rows, width] whose rows are contiguous."""
    if t.dim() != 2 or (like is not None and (t.shape != like.shape or t.dtype != like.dtype)):
        raise ValueError(f"{name}: [rows, width]{'' if like is None else ' like the others'} expected, got {tuple(t.shape)} {t.dtype}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(name: str, t: torch.Tensor, n: int) -> None:
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous float32 values expected, got {tuple(t.shape)} {t.dtype}")


def _out(name: str, t: Optional[torch.Tensor], like: torch.Tensor, dtype=None) -> torch.Tensor:
    """An output [rows, width]: the given one, or a new one."""
    dtype = dtype or like.dtype
    if t is None:
        return torch.empty(like.shape, dtype=dtype, device=like.device)
    if t.shape != like.shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous {tuple(like.shape)} {dtype} expected, got {tuple(t.shape)} {t.dtype}")
    return t


def mtfm_rms_bwd_workspace_bytes(width: int) -> int:
    return int(load_library().mtfm_rms_bwd_workspace_bytes(width))


def _forward(call, x, weight, eps, residual, h, y, rstd, scale, kind):
    n, d = x.shape
    code, x_stride, r_stride = _dtype_code(x), _rows("x", x), 0
    _vector("weight", weight, d)
    if residual is not None:
        r_stride = _rows("residual", residual, x)
        h = _out("h", h, x)
    elif h is not None:
        raise ValueError("h without a residual is x")
    hta.check_on_current_device(x, weight, residual, h, y, rstd, scale)
    P = hta._address
    _call((x.data_ptr(), P(residual), weight.data_ptr(), P(h), y.data_ptr(), P(rstd), P(scale), 0, 0, 0, x_stride, r_stride, 0, n, 0,
           d, eps, code, kind, call))
    return x if h is None else h


def mtfm_rms_fwd(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                 y: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None, save_rstd: bool = True,
                 rstd: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(y, h, rstd) of rows x [n, width] (bf16 or float32) and weight [width] (float32).  h is the sum with the residual (x itself
    without one) and with rstd what the backward pass reads; rstd is None when save_rstd is False.  Outputs may be given, and may
    be the inputs' own memory (y is x, h is residual)."""
    _rows("x", x)
    y = _out("y", y, x)
    if rstd is not None:
        _vector("rstd", rstd, x.shape[0])
    elif save_rstd:
        rstd = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    return y, _forward(_FWD, x, weight, eps, residual, h, y, rstd, None, 0), rstd


def mtfm_rms_fwd_q8(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                    kind: torch.dtype = torch.int8, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                    h: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(q, scale, h) with y = q * scale[:, None] in 8 bits, `kind` torch.int8 or torch.float8_e4m3fn."""
    if kind not in KINDS:
        raise TypeError(f"unsupported 8-bit type {kind}")
    _rows("x", x)
    q = _out("q", q, x, kind)
    if scale is None:
        scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    _vector("scale", scale, x.shape[0])
    return q, scale, _forward(_FWD_Q8, x, weight, eps, residual, h, q, None, scale, KINDS[kind])


def mtfm_rms_bwd(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, dh: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dx, dweight) for the gradients dy of y and dh of h; dx is the gradient of x and of the residual.  `out` may hold preallocated
    (dx, dweight); dx may be dy or dh."""
    code, h_stride = _dtype_code(h), _rows("h", h)
    n, d = h.shape
    dy_stride = _rows("dy", dy, h)
    dh_stride = 0 if dh is None else _rows("dh", dh, h)
    _vector("weight", weight, d)
    _vector("rstd", rstd, n)
    dx, dweight = out or (None, None)
    dx = _out("dx", dx, h)
    if dweight is None:
        dweight = torch.empty_like(weight)
    _vector("dweight", dweight, d)
    if workspace is None:
        workspace = torch.empty(max(mtfm_rms_bwd_workspace_bytes(d), 256), dtype=torch.uint8, device=h.device)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    hta.check_on_current_device(dy, h, weight, rstd, dh, dx, dweight, workspace)
    P = hta._address
    _call((h.data_ptr(), P(dh), weight.data_ptr(), 0, dx.data_ptr(), rstd.data_ptr(), 0, dy.data_ptr(), dweight.data_ptr(),
           workspace.data_ptr(), h_stride, dh_stride, dy_stride, n, workspace.numel() * workspace.element_size(), d, 0.0, code, 0, _BWD))
    return dx, dweight
