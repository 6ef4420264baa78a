"""Layer norm and its gradients (oracle; test infrastructure only), float64.

y = xhat w + b with xhat = (x - mean) / sqrt(var + eps) over a row's channels; weight
and bias [C], or [B, C] with a row per batch entry.  Gradients from given mean and rstd,
as the backward pass takes them.
"""
from __future__ import annotations

import numpy as np


def _rows(w, x, none):
    if w is None:
        return np.full(x.shape[-1], none)
    w = np.asarray(w, dtype=np.float64)
    return w[:, None, :] if w.ndim == 2 else w


def forward(x, weight=None, bias=None, eps=1e-5, unit=0.0):
    """x [B, N, C] -> (y, mean [B, N], rstd [B, N])."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=-1, keepdims=True)
    rstd = 1.0 / np.sqrt(np.mean((x - mean) ** 2, axis=-1, keepdims=True) + eps)
    w = _rows(weight, x, 1.0) + (unit if weight is not None else 0.0)
    return (x - mean) * rstd * w + _rows(bias, x, 0.0), mean[..., 0], rstd[..., 0]


def backward(dy, x, mean, rstd, weight=None, unit=0.0, per_entry=False):
    """(dx, dweight, dbias); the sums over all rows, or with per_entry over an entry's."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    rstd = np.asarray(rstd, dtype=np.float64)[..., None]
    xhat = (x - np.asarray(mean, dtype=np.float64)[..., None]) * rstd
    g = dy * (_rows(weight, x, 1.0) + (unit if weight is not None else 0.0))
    dx = rstd * (g - g.mean(axis=-1, keepdims=True) - xhat * (g * xhat).mean(axis=-1, keepdims=True))
    over = (1,) if per_entry else (0, 1)
    return dx, (dy * xhat).sum(axis=over), dy.sum(axis=over)
