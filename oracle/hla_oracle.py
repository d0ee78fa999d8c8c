"""Float64 oracle of hybrid linear attention with a decay for each head (definition: include/mtfm_hla.h), one token after the
other: the recurrence itself, and its adjoint recurrence backwards.  Test infrastructure only; shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def _users(q_off, kv_off, hist, tgt, full):
    for u in range(len(hist)):
        L, T = int(hist[u]), int(tgt[u])
        kv, q = int(kv_off[u]), int(q_off[u])
        # rows of k (and v), and of q (and out), of the history and of the candidates
        yield u, range(kv, kv + L), range(q, q + L) if full else None, range(kv + L, kv + L + T), range(q + (L if full else 0), q + (L if full else 0) + T)


def decay_of(log_decay):
    g = np.asarray(log_decay, dtype=np.float64)
    return np.exp(np.where(g < 0, g, 0.0))


def forward(q, k, v, log_decay, q_off, kv_off, hist, tgt, scale, full, state=None):
    """(out, states behind the histories); rows of no user stay NaN."""
    Hq, d = q.shape[1:]
    r = Hq // k.shape[1]
    l = decay_of(log_decay)[:, None, None]
    out = np.full(q.shape, np.nan)
    last = np.zeros((len(hist), Hq, d, d))
    for u, h_kv, h_q, t_kv, t_q in _users(q_off, kv_off, hist, tgt, full):
        S = np.zeros((Hq, d, d)) if state is None else state[u].astype(np.float64)
        for i, row in enumerate(h_kv):
            S = l * S + np.repeat(k[row], r, 0)[:, :, None] * np.repeat(v[row], r, 0)[:, None, :]
            if full:
                out[h_q[i]] = scale * np.einsum("hi,hij->hj", q[h_q[i]], S)
        for row, at in zip(t_kv, t_q):
            kk, vv = np.repeat(k[row], r, 0), np.repeat(v[row], r, 0)
            out[at] = scale * (np.einsum("hi,hij->hj", q[at], l * S) + (q[at] * kk).sum(1, keepdims=True) * vv)
        last[u] = S
    return out, last


def backward(dout, q, k, v, log_decay, q_off, kv_off, hist, tgt, scale, full, state=None, dlast=None):
    """(dq, dk, dv, gradient of the first states)."""
    Hq, d = q.shape[1:]
    Hkv = k.shape[1]
    r = Hq // Hkv
    l = decay_of(log_decay)[:, None, None]
    dq, dk, dv = np.full(q.shape, np.nan), np.full(k.shape, np.nan), np.full(k.shape, np.nan)
    first = np.zeros((len(hist), Hq, d, d))
    group = lambda x: x.reshape(Hkv, r, d).sum(1)
    for u, h_kv, h_q, t_kv, t_q in _users(q_off, kv_off, hist, tgt, full):
        S = [np.zeros((Hq, d, d)) if state is None else state[u].astype(np.float64)]
        for row in h_kv:
            S.append(l * S[-1] + np.repeat(k[row], r, 0)[:, :, None] * np.repeat(v[row], r, 0)[:, None, :])
        R = np.zeros((Hq, d, d)) if dlast is None else dlast[u].astype(np.float64)
        for row, at in zip(t_kv, t_q):
            kk, vv = np.repeat(k[row], r, 0), np.repeat(v[row], r, 0)
            R = R + scale * l * q[at][:, :, None] * dout[at][:, None, :]
            own = scale * (dout[at] * vv).sum(1, keepdims=True)
            dq[at] = scale * np.einsum("hij,hj->hi", l * S[-1], dout[at]) + own * kk
            dk[row] = group(own * q[at])
            dv[row] = group(scale * (q[at] * kk).sum(1, keepdims=True) * dout[at])
        for i in reversed(range(len(h_kv))):
            row = h_kv[i]
            if full:
                at = h_q[i]
                R = R + scale * q[at][:, :, None] * dout[at][:, None, :]
                dq[at] = scale * np.einsum("hij,hj->hi", S[i + 1], dout[at])
            dk[row] = group(np.einsum("hij,hj->hi", R, np.repeat(v[row], r, 0)))
            dv[row] = group(np.einsum("hij,hi->hj", R, np.repeat(k[row], r, 0)))
            R = l * R
        first[u] = R
    return dq, dk, dv, first
