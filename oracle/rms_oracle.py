"""Float64 oracle of the root-mean-square normalization (definition: include/mtfm_rms.h).  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def forward(h, weight, eps):
    """(y, rstd) of rows h."""
    h = h.astype(np.float64)
    rstd = 1.0 / np.sqrt((h * h).sum(1) / h.shape[1] + eps)
    return h * rstd[:, None] * weight, rstd


def backward(dy, h, weight, eps, dh=None):
    """(dx, dweight), and the sums of the magnitudes that either is a difference or sum of."""
    h, dy = h.astype(np.float64), dy.astype(np.float64)
    rstd = 1.0 / np.sqrt((h * h).sum(1) / h.shape[1] + eps)
    xhat, w = h * rstd[:, None], dy * weight
    dx = rstd[:, None] * (w - xhat * (w * xhat).mean(1, keepdims=True))
    size = rstd[:, None] * (np.abs(w) + np.abs(xhat) * np.abs(w * xhat).mean(1, keepdims=True))
    if dh is not None:
        dx, size = dx + dh, size + np.abs(dh)
    return dx, (dy * xhat).sum(0), size, np.abs(dy * xhat).sum(0)
