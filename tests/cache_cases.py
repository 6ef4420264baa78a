"""Inputs and bounds shared by the GPU tests of the cache operators: a cache filled
on the host, and attention over it by oracle/kv_cache.py."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import kv_cache as okv

BF16, F32 = torch.bfloat16, torch.float32
CODES = {"bf16": BF16, "e4m3": torch.uint8, "int8": torch.int8}


def bf16_normal(g, shape, scale=1.0):
    """N(0, scale^2) values that bf16 holds, as a host tensor."""
    return torch.from_numpy(g.standard_normal(shape).astype(np.float32) * np.float32(scale)).to(BF16)


def host_cache(g, pages, kv, page, dim, fmt, scale=1.0):
    """A cache on the host with every slot filled, and its K and V in float64 [pages, kv, page, D]."""
    shape = (pages, kv, page, dim)
    cache, values = {}, {}
    for n in ("k", "v"):
        if fmt == "bf16":
            cache[n] = bf16_normal(g, shape, scale)
            cache[n + "_scale"] = None
            values[n] = cache[n].double().numpy()
            continue
        s = np.exp(g.uniform(-1, 1, shape[:3])).astype(np.float32) * np.float32(scale)
        if fmt == "e4m3":
            s = np.exp2(np.round(np.log2(s))).astype(np.float32) * np.float32(2.0 ** -8)
            codes = g.integers(0, 256, shape).astype(np.uint8)
            codes[(codes & 0x7F) == 0x7F] -= 1              # no NaN
            cache[n] = torch.from_numpy(codes)
            values[n] = okv.e4m3_values()[codes]
        else:
            s = s / np.float32(64)
            codes = g.integers(-127, 128, shape).astype(np.int8)
            cache[n] = torch.from_numpy(codes)
            values[n] = codes.astype(np.float64)
        cache[n + "_scale"] = torch.from_numpy(s)
        values[n] = values[n] * s.astype(np.float64)[..., None]
    return cache, values


def to_gpu(cache):
    return {n: None if x is None else x.cuda() for n, x in cache.items()}


def rows_of(values, n, table, length, page, head, num_pages):
    """K or V rows [length, D] of one entry's head, and which of them exist (bad pages do not)."""
    at = np.arange(length)
    pages = np.asarray(table)[at // page]
    ok = (pages >= 0) & (pages < num_pages)
    return values[n][np.where(ok, pages, 0), head, at % page], ok


def attend(values, q, table, lengths, page, k_new=None, v_new=None, mask=None, counts=None, scale=None):
    """oracle/kv_cache.py over every entry and head.  Returns out, lse (float64) and
    the scale of their rounding errors: per row sum_j w_j |v_jd| [B, H, T, D], and the
    largest sum_d |q_d k_jd| of a seen key [B, H, T] times the softmax scale."""
    q = q.double().numpy()
    B, H, T, D = q.shape
    num_pages, kv = values["k"].shape[:2]
    G = H // kv
    c = 1.0 / math.sqrt(D) if scale is None else scale
    out, lse = np.zeros((B, H, T, D)), np.full((B, H, T), -np.inf)
    size, dot = np.zeros((B, H, T, D)), np.zeros((B, H, T))
    for b in range(B):
        cap = table.shape[1] * page
        n = int(np.clip(lengths[b], 0, cap))
        cnt = T if counts is None else int(np.clip(counts[b], 0, T))
        for h in range(kv):
            k, ok = rows_of(values, "k", table[b], n, page, h, num_pages)
            v, _ = rows_of(values, "v", table[b], n, page, h, num_pages)
            seen = np.tile(ok, (cnt, 1))
            if k_new is not None:
                k = np.concatenate([k, k_new[b, h, :cnt].double().numpy()])
                v = np.concatenate([v, v_new[b, h, :cnt].double().numpy()])
                m = np.tril(np.ones((cnt, cnt), bool)) if mask is None else (mask[b] if mask.ndim == 3 else mask)[:cnt, :cnt] != 0
                seen = np.concatenate([seen, m], axis=1)
            for i in range(h * G, (h + 1) * G):
                out[b, i, :cnt], lse[b, i, :cnt] = okv.attention(q[b, i, :cnt], k, v, seen, c)
                for t in range(cnt):
                    at = np.flatnonzero(seen[t])
                    if at.size:
                        s = c * (k[at] @ q[b, i, t])
                        w = np.exp(s - lse[b, i, t])
                        with np.errstate(invalid="ignore"):
                            size[b, i, t] = w @ np.abs(v[at])
                        dot[b, i, t] = (c * np.abs(k[at]) @ np.abs(q[b, i, t])).max()
    return out, lse, size, dot


def bounds(out, lse, size, dot, keys, dim, f32):
    """How far the kernel's results may be from float64's, counted in roundings:
    a logit is D products added in float32 and three more products (scales, base 2):
    (D + 8) half steps of sum |q k|; a weight then errs by that, 4 half steps of the
    exponential and its argument, and, before the product with V, half a step of bf16
    (bf16 result) or of its square (float32 result, two bf16 parts); numerator and
    sum add up to `keys` terms in float32; the division and the result round once
    each."""
    h32, h16 = 2.0 ** -24, 2.0 ** -8
    logit = (dim + 8) * h32 * dot
    weight = logit + (8 + keys) * h32
    part = h16 * h16 * 2 if f32 else h16
    o = size * (part + 2 * weight[..., None]) + np.abs(out) * (2 * h32 + (0 if f32 else h16)) + 1e-30
    with np.errstate(invalid="ignore"):
        e = logit + (8 + keys) * h32 + 4 * h32 * np.where(np.isfinite(lse), np.abs(lse), 0)
    return o, e


def check(got, got_lse, want, keys, dim, f32=False, rows=None):
    out, lse, size, dot = want
    o_tol, l_tol = bounds(out, lse, size, dot, keys, dim, f32)
    got = got.double().cpu().numpy()
    on = np.ones(out.shape[:3], bool) if rows is None else rows
    err = np.abs(got - out)
    worst = (err / o_tol)[on].max() if on.any() else 0.0
    assert np.isfinite(got[on]).all() and worst <= 1.0, worst
    if got_lse is not None:
        x = got_lse.double().cpu().numpy()
        fin = np.isfinite(lse) & on
        assert np.array_equal(np.isneginf(x)[on], np.isneginf(lse)[on])
        assert (np.abs(x - lse)[fin] <= l_tol[fin]).all()
    return worst
