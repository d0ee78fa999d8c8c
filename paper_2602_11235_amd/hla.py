"""Thin ctypes binding of hybrid linear attention with a decay for each head (C ABI declared in include/mtfm_hla.h): a user's
history as a d x d state per query head, S <- exp(log_decay) S + k v^T, o = scale q S; candidates see the history's state and
themselves.  Argument checks and marshalling only; PyTorch supplies device memory and the stream; no fallback without the library."""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

import torch

from . import hta

EXPORTS = ("mtfm_hla_workspace_bytes", "mtfm_hla_fwd", "mtfm_hla_bwd", "mtfm_hla_step")
KERNEL_FWD, KERNEL_STATES, KERNEL_BWD, KERNEL_SUM, KERNEL_STEP = 10, 11, 12, 13, 14

_declared = None

# argument blocks of mtfm_binding_hla and mtfm_binding_hla_step (struct HlaArgs, HlaStepArgs of csrc/binding.hip), see hta.call_packed
_BLOCK = struct.Struct("18P3q6if3i")
_STEP_BLOCK = struct.Struct("8P5if2i")


def load_library() -> ctypes.CDLL:
    global _declared
    if _declared is not None:
        return _declared
    lib = hta.load_library()
    vp, i32, i64, f32, sz, ci = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t,
                                 ctypes.c_int)
    lib.mtfm_hla_workspace_bytes.restype = sz
    lib.mtfm_hla_workspace_bytes.argtypes = [ci, ci, ci, i32, i64, i64, i32, i32, i32, i32, i32]
    tail = [vp] * 4 + [i32, i64, i64, i32, i32, i32, i32, i32, f32, ci, ci, vp, sz, vp]
    lib.mtfm_hla_fwd.restype = ci
    lib.mtfm_hla_fwd.argtypes = [vp] * 7 + tail
    lib.mtfm_hla_bwd.restype = ci
    lib.mtfm_hla_bwd.argtypes = [vp] * 11 + tail
    lib.mtfm_hla_step.restype = ci
    lib.mtfm_hla_step.argtypes = [vp] * 8 + [i32, i32, i32, i32, i32, f32, ci, vp]
    for fn in (lib.mtfm_binding_hla, lib.mtfm_binding_hla_step):
        fn.restype = ci
        fn.argtypes = [vp, vp]
    _declared = lib
    return lib


def mtfm_hla_workspace_bytes(layer, dtype, is_bwd, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, head_dim) -> int:
    n = load_library().mtfm_hla_workspace_bytes(layer, dtype, int(is_bwd), batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv,
                                                head_dim)
    if n == ctypes.c_size_t(-1).value:
        raise hta.HtaError(hta.ERR_INVALID_ARG, hta.mtfm_hta_last_error())
    return int(n)


def _check(name: str, t: torch.Tensor, shape, dtype) -> None:
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous {tuple(shape)} {dtype} expected, got {tuple(t.shape)} {t.dtype}")


def _check_tokens(q, k, v) -> None:
    if q.dim() != 3 or k.dim() != 3 or k.shape[2] != q.shape[2]:
        raise ValueError(f"q [rows, Hq, head_dim] and k [rows, Hkv, head_dim] expected, got {tuple(q.shape)} and {tuple(k.shape)}")
    for name, t, like in (("q", q, q), ("k", k, k), ("v", v, k)):
        _check(name, t, like.shape, torch.bfloat16)


class DecayBatch:
    """Device buffers of one jagged batch (allocation and marshalling only); arguments as for hta.Batch, without a softmax.

    log_decay [Hq] float32; state: S_0 [batch, Hq, head_dim, head_dim] float32 or None (zero); want_state: forward() returns the states
    behind the histories too.  Results live in buffers of the batch, which the next call of the same kind overwrites."""

    def __init__(self, q, k, v, log_decay, q_offsets, kv_offsets, hist_len, n_targets, max_hist, max_targets, scale, layer,
                 state: Optional[torch.Tensor] = None, want_state: bool = False):
        _check_tokens(q, k, v)
        batch, Hq, d = int(hist_len.shape[0]), int(q.shape[1]), int(q.shape[2])
        _check("log_decay", log_decay, (Hq,), torch.float32)
        for name, t, n in (("q_offsets", q_offsets, batch + 1), ("kv_offsets", kv_offsets, batch + 1), ("hist_len", hist_len, batch),
                           ("n_targets", n_targets, batch)):
            _check(name, t, (n,), torch.int32)
        self._state_shape = (batch, Hq, d, d)
        if state is not None:
            _check("state", state, self._state_shape, torch.float32)
        hta.check_on_current_device(q, k, v, log_decay, q_offsets, kv_offsets, hist_len, n_targets, state)
        self.q, self.k, self.v, self.log_decay, self.state = q, k, v, log_decay, state
        self.ints = (q_offsets, kv_offsets, hist_len, n_targets)
        self.scale, self.layer = float(scale), int(layer)
        self.total_q, self.total_kv = int(q.shape[0]), int(k.shape[0])
        self.sizes = (batch, int(max_hist), int(max_targets), Hq, int(k.shape[1]), d)
        self.fwd_workspace = self._workspace(False)
        self.out = torch.empty_like(q)
        self.final_state = torch.empty(self._state_shape, dtype=torch.float32, device=q.device) if want_state else None
        self.dq = self.dk = self.dv = self.dstate = self.bwd_workspace = None

    def _workspace(self, is_bwd: bool) -> Optional[torch.Tensor]:
        batch, *rest = self.sizes
        n = mtfm_hla_workspace_bytes(self.layer, hta.BF16, is_bwd, batch, self.total_q, self.total_kv, *rest)
        return torch.empty(n, dtype=torch.uint8, device=self.q.device) if n else None

    def _call(self, dout, dfinal, workspace, stream) -> None:
        back = dout is not None
        hta.check_on_current_device(self.q, dout, dfinal)
        P = hta._address
        grads = (dout.data_ptr(), self.dq.data_ptr(), self.dk.data_ptr(), self.dv.data_ptr(), P(dfinal), P(self.dstate)) if back else (0,) * 6
        q_offsets, kv_offsets, hist_len, n_targets = self.ints
        status = (_declared or load_library()).mtfm_binding_hla(_BLOCK.pack(
            self.q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), self.out.data_ptr(), self.log_decay.data_ptr(), P(self.state),
            P(self.final_state), *grads, q_offsets.data_ptr(), kv_offsets.data_ptr(), hist_len.data_ptr(), n_targets.data_ptr(), P(workspace),
            0 if workspace is None else workspace.numel(), self.total_q, self.total_kv, *self.sizes, self.scale, hta.BF16, self.layer, back),
            hta._stream_handle(stream))
        if status != hta.OK:
            raise hta.HtaError(status, hta.mtfm_hta_last_error())

    def forward(self, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """(out, the states behind the histories or None)."""
        self._call(None, None, self.fwd_workspace, stream)
        return self.out, self.final_state

    def prepare_backward(self) -> None:
        if self.dq is None:
            self.bwd_workspace = self._workspace(True)
            if self.state is not None:
                self.dstate = torch.empty_like(self.state)
            self.dk, self.dv = torch.empty_like(self.k), torch.empty_like(self.v)
            self.dq = torch.empty_like(self.q)

    def backward(self, dout, dstate: Optional[torch.Tensor] = None, stream=None):
        """(dq, dk, dv, gradient of `state` or None) for the gradient of out and, optionally, `dstate` of the states behind the
        histories.  Does not need forward() to have run."""
        _check("dout", dout, self.q.shape, torch.bfloat16)
        if dstate is not None:
            _check("dstate", dstate, self._state_shape, torch.float32)
        self.prepare_backward()
        self._call(dout, dstate, self.bwd_workspace, stream)
        return self.dq, self.dk, self.dv, self.dstate


def mtfm_hla_step(q, k, v, state, slots, log_decay, scale, new_state=None, out=None, stream=None) -> torch.Tensor:
    """One history token per row: q [rows, Hq, d], k, v [rows, Hkv, d]; row i's state is slot slots[i] (int32; None: i) of the pool
    `state` [slots, Hq, d, d] float32, and what follows goes to the same slot of `new_state` (None: in place).  Rows of one slot are
    tokens in the order of the rows; a row whose slot is not in the pool is padding, with output zero.  Returns out like q."""
    # (one condition for all that is right: a call is worth a few microseconds, and each look at a tensor a tenth of one; what is wrong is said by _check)
    qs, ks, ss, bf16, f32 = q.shape, k.shape, state.shape, torch.bfloat16, torch.float32
    if not (len(qs) == 3 and len(ks) == 3 and ks[0] == qs[0] and ks[2] == qs[2] and len(ss) == 4 and ss[1] == qs[1] and ss[2] == ss[3] == qs[2]
            and v.shape == ks and q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and state.dtype is f32
            and q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and state.is_contiguous()):
        _check_tokens(q, k, v)
        _check("k", k, (qs[0], *ks[1:]), bf16)
        _check("state", state, (*ss[:1], *qs[1:], qs[2]), f32)
    rows, Hq, d = qs
    if new_state is None:
        new_state = state
    elif new_state.shape != ss or new_state.dtype is not f32 or not new_state.is_contiguous():
        _check("new_state", new_state, ss, f32)
    if slots is not None and (slots.dim() != 1 or slots.shape[0] != rows or slots.dtype is not torch.int32 or not slots.is_contiguous()):
        _check("slots", slots, (rows,), torch.int32)
    if log_decay.dim() != 1 or log_decay.shape[0] != Hq or log_decay.dtype is not f32 or not log_decay.is_contiguous():
        _check("log_decay", log_decay, (Hq,), f32)
    if out is None:
        out = torch.empty_like(q)
    else:
        _check("out", out, qs, bf16)
    hta.check_on_current_device(q, k, v, state, slots, log_decay, new_state, out)
    status = (_declared or load_library()).mtfm_binding_hla_step(_STEP_BLOCK.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), state.data_ptr(), new_state.data_ptr(), hta._address(slots),
        out.data_ptr(), rows, ss[0], Hq, ks[1], d, scale, hta.BF16, 0), hta._stream_handle(stream))
    if status != hta.OK:
        raise hta.HtaError(status, hta.mtfm_hta_last_error())
    return out
