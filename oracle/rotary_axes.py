"""Rotary positions on several axes (oracle; test infrastructure only), float64.

The pairs of an axis of n pairs turn by position * base^(-j / n), j < n; axes follow each
other.  Pair i of a row, as the complex number a + ib, is multiplied by exp(i angle).
"""
from __future__ import annotations

import numpy as np

from . import rotary


def ladders(sections, base=10000.0, **kw):
    """(frequencies of all pairs, axis of each pair, magnitude); base and the scalings of
    rotary.frequencies for all axes, or one of each per axis."""
    freq, axis, mags = [], [], []
    for a, n in enumerate(sections):
        pick = {k: v[a] if isinstance(v, (list, tuple)) else v for k, v in dict(kw, base=base).items()}
        f, m = rotary.frequencies(2 * n, **pick)
        freq.append(f)
        axis += [a] * n
        mags.append(m)
    return np.concatenate(freq), np.array(axis), mags[0]


def apply(x, positions, freq, axis, magnitude, layout, backward=False):
    """x [B, H, N, D], positions [B, N, axes] -> float64."""
    x = np.asarray(x, dtype=np.float64)
    pairs = len(freq)
    p = np.asarray(positions, dtype=np.float64)
    known = (axis >= 0) & (axis < p.shape[-1])
    phi = np.where(known, p[..., np.where(known, axis, 0)], 0.0)[:, None] * freq
    z = magnitude * np.exp(-1j * phi if backward else 1j * phi)
    out = x.copy()
    first, second = ((slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "half"
                     else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)))
    w = (x[..., first] + 1j * x[..., second]) * z
    out[..., first], out[..., second] = w.real, w.imag
    return out
