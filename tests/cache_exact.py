"""Inputs for the attention over a cache whose float32 arithmetic is exact, or almost:
a lost, repeated or misplaced key shows as more than a rounding, and so does a weight
with fewer bits than it should have.  With what the results may be off by.

whole_case: logits of base 2 are whole numbers in {-1, 0, 1} (softmax scale ln 2: c log2(e) is
1 in float32), so weights and rescalings are powers of two; values are whole numbers up to
8.  Every product and sum is then a multiple of 1/4 far below 2^22, exact in float32 whatever
its order, and the weights fit bf16.  Left are the reciprocal of the sum and the product with
it, two half steps of float32, and a bf16 result's own rounding.

fine_case: QK^T is a whole number (exact in float32), the scales on it are not, logits of base 2
are within +-2, values are normal.  Errors of float32 results in half steps u = 2^-24, root mean
squares of independent roundings (a rounding's is 0.41 of its largest).  A weight: the scale's
rounding and the argument's, 1.4 and 2.8 at most through ln 2; the exponential, 2; the product with
V's scale and what three bf16 parts leave, 1 each: 1.6 in all, say 2.  The denominator, of up to 500
keys in one run or nine parts: a chain of up to 132 additions (128 in a lane, then lanes and waves, or 32
and 3 for each part), 0.41 sqrt(132) = 4.7.  The numerator: up to 48 matrix products in a chain, 0.7 of
the accumulator each (as measured on one), which grows along it: 0.7 sqrt(48 / 2) = 3.4.  Together
6.2 u = 3.7e-7 of the results' norm; three times that is allowed.
Weights of two bf16 parts are off by 2.3e-6 and more (tests/test_cache_exact.py).
"""
from __future__ import annotations

import math

import numpy as np
import torch

BF16 = torch.bfloat16
LN2 = math.log(2.0)
U = 2.0 ** -24
FINE_NORM = 3 * 6.2 * U


def _cache(g, pages, kv, page, dim, fmt, k_values, v_values, scales):
    """(cache, K and V in float64): rows k_values / v_values (what the codes say) times scales [pages, kv, page]."""
    cache, values = {}, {}
    for n, x in (("k", k_values), ("v", v_values)):
        if fmt == "bf16":
            cache[n], cache[n + "_scale"] = torch.from_numpy(x.astype(np.float32)).to(BF16), None
            values[n] = cache[n].double().numpy()
            continue
        t = torch.from_numpy(x.astype(np.float32))
        cache[n] = t.to(torch.float8_e4m3fn).view(torch.uint8) if fmt == "e4m3" else t.round().to(torch.int8)
        codes = cache[n].view(torch.float8_e4m3fn).double() if fmt == "e4m3" else cache[n].double()
        cache[n + "_scale"] = torch.from_numpy(scales[n].astype(np.float32))
        values[n] = codes.numpy() * cache[n + "_scale"].double().numpy()[..., None]
    return cache, values


class Inputs:
    """One call: a cache behind shuffled pages, queries, drafted keys and values, a mask, counts."""

    def __init__(self, g, B, kv, G, T, D, page, fmt, lengths, pool=0):
        self.g, self.B, self.kv, self.G, self.T, self.D, self.page, self.fmt = g, B, kv, G, T, D, page, fmt
        self.lengths = np.array(lengths, dtype=np.int32)
        P = max(1, -(-int(max(lengths)) // page))
        self.pages = pool or B * P + 1
        self.table = (g.integers(0, pool, (B, P)) if pool else           # pages that entries share
                      g.permutation(self.pages)[:B * P].reshape(B, P)).astype(np.int32)
        m = np.tril(g.random((B, T, T)) < 0.5).astype(np.uint8)
        m[:, np.arange(T), np.arange(T)] = 1
        self.mask = m
        self.counts = np.array([T] + [max(1, T - 1 - b % 3) for b in range(1, B)], dtype=np.int32)

    def rows(self, n, b, h):
        at = np.arange(int(self.lengths[b]))
        return self.values[n][self.table[b][at // self.page], h, at % self.page]

    def exact(self):
        """Results in float64 [B, H, T, D], lse [B, H, T], and which rows exist."""
        B, H, T, D = self.B, self.kv * self.G, self.T, self.D
        out, lse, here = np.zeros((B, H, T, D)), np.zeros((B, H, T)), np.zeros((B, H, T), bool)
        q, kn, vn = (x.double().numpy() for x in (self.q, self.k_new, self.v_new))
        for b in range(B):
            n, c = int(self.lengths[b]), int(self.counts[b])
            here[b, :, :c] = True
            seen = np.ones((c, n + c), bool)
            seen[:, n:] = self.mask[b, :c, :c] != 0
            for h in range(self.kv):
                k = np.concatenate((self.rows("k", b, h), kn[b, h, :c]))
                v = np.concatenate((self.rows("v", b, h), vn[b, h, :c]))
                for i in range(h * self.G, (h + 1) * self.G):
                    s = np.where(seen, self.scale * (q[b, i, :c] @ k.T), -np.inf)
                    top = s.max(axis=1, keepdims=True)
                    w = np.exp(s - top)
                    out[b, i, :c] = w @ v / w.sum(axis=1, keepdims=True)
                    lse[b, i, :c] = top[:, 0] + np.log(w.sum(axis=1))
        return out, lse, here


def whole_case(seed, B, kv, G, T, D, page, fmt, lengths, pool=0):
    g = np.random.default_rng(seed)
    c = Inputs(g, B, kv, G, T, D, page, fmt, lengths, pool)
    rows = (c.pages, kv, page)
    scales = {n: np.exp2(g.integers(-1, 1, rows)) for n in ("k", "v")}
    one = {n: np.ones(rows) if fmt == "bf16" else scales[n] for n in ("k", "v")}
    k = g.integers(-3, 4, rows + (D,)).astype(np.float64)            # what Q does not look at
    k[..., 0] = g.integers(0, 2, rows) / one["k"]                    # 0 or 1 after its scale
    v = g.integers(-8, 9, rows + (D,)) / one["v"][..., None]
    c.cache, c.values = _cache(g, c.pages, kv, page, D, fmt, k, v, scales)
    q = np.zeros((B, kv * G, T, D))
    q[..., 0] = g.integers(-1, 2, (B, kv * G, T))
    kn = g.integers(-3, 4, (B, kv, T, D)).astype(np.float64)
    kn[..., 0] = g.integers(0, 2, (B, kv, T))
    c.q, c.k_new, c.v_new = (torch.from_numpy(x.astype(np.float32)).to(BF16)
                             for x in (q, kn, g.integers(-8, 9, (B, kv, T, D))))
    c.scale = LN2
    return c


def fine_case(seed, B, kv, G, T, D, page, fmt, lengths):
    g = np.random.default_rng(seed)
    c = Inputs(g, B, kv, G, T, D, page, fmt, lengths)
    rows = (c.pages, kv, page)
    # 16 channels of q in [-3, 3] meet k in [-7, 7]: |S| <= 336; scales in [1/2, 1]
    scales = {"k": g.uniform(0.5, 1.0, rows) if fmt == "int8" else np.exp2(g.integers(-1, 1, rows)),
              "v": g.uniform(0.5, 1.0, rows) / 32 if fmt == "int8" else np.exp2(g.integers(-1, 1, rows) - 4.0)}
    k = g.integers(-7, 8, rows + (D,)).astype(np.float64)
    v = g.standard_normal(rows + (D,)) * (1.0 if fmt == "bf16" else 32.0)
    c.cache, c.values = _cache(g, c.pages, kv, page, D, fmt, k, np.clip(v, -127, 127), scales)
    q = np.zeros((B, kv * G, T, D))
    q[..., :16] = g.integers(-3, 4, (B, kv * G, T, 16))
    kn = g.integers(-7, 8, (B, kv, T, D))
    c.q, c.k_new, c.v_new = (torch.from_numpy(x.astype(np.float32)).to(BF16)
                             for x in (q, kn, g.standard_normal((B, kv, T, D))))
    c.scale = 2.0 / 336 * LN2                                        # |base-2 logits| <= 2
    return c


def check_whole(got, lse, want, f32):
    out, wl, here = want
    x = got.double().cpu().numpy()[here] if isinstance(got, torch.Tensor) else got[here]
    y = out[here]
    tol = np.abs(y) * (2.001 * U + (0.0 if f32 else 2.0 ** -8)) + 1e-13      # (1e-13: the oracle's own sums)
    worst = np.abs(x - y) - tol
    assert np.isfinite(x).all() and (worst <= 0).all(), (int((worst > 0).sum()), float(np.abs(x - y).max()))
    if lse is not None:
        z = lse.double().cpu().numpy()[here]
        # log2 of the sum (2 half steps of at most 16), its sum with the reference, times ln 2, which is rounded
        assert (np.abs(z - wl[here]) <= 8 * U * np.maximum(np.abs(wl[here]), 1.0)).all()


def norm_error(got, want):
    out, _, here = want
    x = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    return float(np.linalg.norm(x[here] - out[here]) / np.linalg.norm(out[here]))
