"""Quantised key/value cache and attention over it (oracle; test infrastructure
only), float64 and from the definitions.

Row formats: e4m3 with scale 2^e, the smallest e in [-127, 127] with max|x| <=
448 * 2^e (0 for a zero row); int8 with scale float32(max|x| / 127), 1 where that
is zero; codes are the nearest values, ties to the even code.  Attention: the
softmax over the keys that a query sees, and nothing else.
"""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """The 256 codes' values (OCP e4m3: bias 7, no infinities, code 0x7f NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = math.nan if (c & 0x7F) == 0x7F else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out[c] = -v if c >= 128 else v
    return out


_VALUES = e4m3_values()
_POSITIVE = _VALUES[:127]                          # ascending


def round_e4m3(x) -> np.ndarray:
    """Nearest e4m3 values of |x| <= 448 by search in the table, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.copysign(_POSITIVE[code], x)


def quantise_rows(x, fmt):
    """(values of the codes, scales) of rows x [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    top = np.abs(x).max(axis=-1)
    if fmt == "e4m3":
        scale = np.ones_like(top)
        for at in np.ndindex(top.shape):
            if top[at] > 0:
                e = -127
                while top[at] > 448.0 * 2.0 ** e and e < 127:
                    e += 1
                scale[at] = 2.0 ** e
        return round_e4m3(x / scale[..., None]), scale
    if fmt == "int8":
        scale = (top / 127.0).astype(np.float32).astype(np.float64)
        scale[scale == 0] = 1.0
        return np.clip(np.rint(x / scale[..., None]), -127, 127), scale
    raise ValueError(fmt)


def attention(q, k_rows, v_rows, seen, scale):
    """q [R, D]; k_rows, v_rows [L, D]; seen [R, L] -> (out [R, D], lse [R])."""
    out = np.zeros((q.shape[0], v_rows.shape[1]))
    lse = np.full(q.shape[0], -np.inf)
    for r in range(q.shape[0]):
        at = np.flatnonzero(seen[r])
        if at.size == 0:
            continue
        s = scale * (k_rows[at] @ q[r])
        m = s.max()
        w = np.exp(s - m)
        lse[r] = m + math.log(w.sum())
        out[r] = (w / w.sum()) @ v_rows[at]
    return out, lse
