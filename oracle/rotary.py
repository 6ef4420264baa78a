"""1-D rotary positions (oracle; test infrastructure only), float64.

Pair i of a row at position p, as the complex number a + ib, is multiplied by
m exp(i p f_i) (its gradient by the conjugate).  Frequencies f_i =
base^(-2i/r); scaled by a factor s: linear f/s; NTK base * s^(r/(r-2)); YaRN
(Peng et al. 2023, "by parts"): g f + (1 - g) f/s with g the clamped ramp of the
turns over the trained context between beta_slow and beta_fast, m = 0.1 ln s + 1.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_len=0.0, beta_fast=32.0, beta_slow=1.0,
                magnitude=0.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "ntk" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = np.exp(-2.0 * i / rot * math.log(base))
    m = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "yarn":
        turns = original_len * f / (2 * math.pi)
        g = np.clip((turns - beta_slow) / (beta_fast - beta_slow), 0, 1)
        f = g * f + (1 - g) * f / factor
        m = 0.1 * math.log(factor) + 1.0
    return f, (magnitude if magnitude > 0 else m)


def apply(x, positions, freq, magnitude, layout, backward=False):
    """x [B, H, N, D], positions [B, N] integers -> float64."""
    x = np.asarray(x, dtype=np.float64)
    rot = 2 * len(freq)
    phi = np.asarray(positions, dtype=np.float64)[:, None, :, None] * freq
    z = magnitude * np.exp(-1j * phi if backward else 1j * phi)
    out = x.copy()
    first, second = ((slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half"
                     else (slice(0, rot, 2), slice(1, rot, 2)))
    w = (x[..., first] + 1j * x[..., second]) * z
    out[..., first], out[..., second] = w.real, w.imag
    return out
