"""Cross attention and its gradients (oracle; test infrastructure only), float64.

softmax(c Q K^T) V over the keys that `seen` [B, M] allows; head h reads kv head
h / (H / Hkv); zeros and -inf where no key is seen.  Gradients from given out and lse, as
the backward pass takes them.  Hidden keys are left out before any arithmetic.
"""
from __future__ import annotations

import numpy as np


def seen_keys(B, M, lengths=None, mask=None):
    seen = np.ones((B, M), dtype=bool)
    if lengths is not None:
        seen &= np.arange(M) < np.asarray(lengths)[:, None]
    if mask is not None:
        seen &= np.asarray(mask) != 0
    return seen


def forward(q, k, v, seen, c):
    """(out [B, H, N, D], lse [B, H, N])."""
    B, H, N, D = q.shape
    group = H // k.shape[1]
    out, lse = np.zeros((B, H, N, D)), np.full((B, H, N), -np.inf)
    for b in range(B):
        at = np.flatnonzero(seen[b])
        if len(at) == 0:
            continue
        for h in range(H):
            s = c * (q[b, h] @ k[b, h // group, at].T)
            top = s.max(axis=-1, keepdims=True)
            p = np.exp(s - top)
            total = p.sum(axis=-1, keepdims=True)
            out[b, h] = (p / total) @ v[b, h // group, at]
            lse[b, h] = (top + np.log(total))[:, 0]
    return out, lse


def backward(dout, q, k, v, out, lse, seen, c):
    """(dq, dk, dv)."""
    B, H, N, D = q.shape
    group = H // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        at = np.flatnonzero(seen[b])
        if len(at) == 0:
            continue
        for h in range(H):
            kv = h // group
            kk, vv = k[b, kv, at], v[b, kv, at]
            p = np.exp(c * (q[b, h] @ kk.T) - lse[b, h][:, None])
            ds = p * (dout[b, h] @ vv.T - (dout[b, h] * out[b, h]).sum(axis=-1, keepdims=True))
            dq[b, h] = c * ds @ kk
            dk[b, kv, at] += c * ds.T @ q[b, h]
            dv[b, kv, at] += p.T @ dout[b, h]
    return dq, dk, dv
