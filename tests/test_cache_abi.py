"""Refusals of the rotary, cache and cache-attention entry points, before any HIP
call: the C ABI with addresses that are never dereferenced, and the binding with
host tensors."""
import ctypes
import math

import pytest

import paper_2606_23743_amd as sva
from oracle import rotary as orot
from paper_2606_23743_amd import _lib
from paper_2606_23743_amd._lib import Cache, CacheQuery, Heads, RotaryParams, RotarySpec

pytestmark = pytest.mark.cpu

torch = pytest.importorskip("torch")

A, MB = 1 << 30, 1 << 24
OK, BAD, SHAPE, ALIGN, UNSUP = (_lib.SVA_OK, _lib.SVA_ERR_INVALID_ARG, _lib.SVA_ERR_SHAPE, _lib.SVA_ERR_ALIGNMENT,
                                _lib.SVA_ERR_UNSUPPORTED)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def heads(at, h, n, d, token_major=False, b=1):
    sh, sn = (d, h * d) if token_major else (n * d, d)
    return Heads(at, h, h * n * d, sh, sn)


def test_new_symbols_are_declared():
    assert set(_lib.header_functions()) >= {"sva_rotary_frequencies", "sva_rotary", "sva_cache_write", "sva_cache_read",
                                            "sva_cache_attention_workspace", "sva_cache_attention"}


@pytest.mark.parametrize("kw", [dict(rot=64), dict(rot=2, scaling="ntk", factor=4.0), dict(rot=62, scaling="linear", factor=3.0),
                                dict(rot=128, scaling="ntk", factor=8.0, base=500000.0),
                                dict(rot=128, scaling="yarn", factor=16.0, original_len=4096),
                                dict(rot=64, scaling="yarn", factor=2.5, original_len=32768, beta_fast=8.0, beta_slow=0.0,
                                     magnitude=0.7)])
def test_frequencies_match_the_oracle(kw):
    want, m = orot.frequencies(**kw)
    kw = dict(kw)
    got, mag = sva.rotary_frequencies(kw.pop("rot"), **kw)
    # both are float64: a few roundings of pow and exp
    assert len(got) == len(want) and max(abs(a / b - 1) for a, b in zip(got, want)) < 1e-13
    assert math.isclose(mag, m, rel_tol=1e-15)


def test_frequencies_refusals(lib):
    buf, mag = (ctypes.c_double * 512)(), ctypes.c_double()
    good = dict(rot_dim=64, scaling=3, base=1e4, factor=2.0, original_len=4096.0, beta_fast=32.0, beta_slow=1.0,
                magnitude=0.0)
    call = lambda **kw: lib.sva_rotary_frequencies(RotarySpec(**{**good, **kw}), buf, mag)  # noqa: E731
    assert call() == OK
    nan, inf = math.nan, math.inf
    for kw in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=514), dict(scaling=4), dict(scaling=-1), dict(base=1.0),
               dict(base=nan), dict(factor=0.5), dict(factor=inf), dict(original_len=0.0), dict(beta_fast=1.0),
               dict(beta_slow=-1.0), dict(magnitude=nan), dict(scaling=2, factor=1e300, base=1e300)):
        assert call(**kw) == BAD, kw
    assert call(scaling=0, factor=0.0, original_len=0.0) == OK      # not read without scaling
    assert lib.sva_rotary_frequencies(None, buf, mag) == BAD


def test_rotary_refusals(lib):
    B, H, N, D = 2, 4, 8, 64
    good = dict(batch=B, tokens=N, head_dim=D, rot_dim=D, layout=0, dtype=0, backward=0, magnitude=1.0)

    def call(qi=None, qo=None, ki=None, ko=None, freq=A, pos=A, pos_b=N, k=True, **kw):
        qi = qi or heads(A, H, N, D)
        qo = qo or heads(A + MB, H, N, D)
        if k:
            ki, ko = ki or heads(A + 2 * MB, 2, N, D), ko or heads(A + 3 * MB, 2, N, D)
        return lib.sva_rotary(RotaryParams(**{**good, **kw}), freq, pos, pos_b, qi, qo, ki, ko, None)

    for kw in (dict(batch=0), dict(tokens=0), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=66), dict(layout=2),
               dict(dtype=2), dict(magnitude=math.nan), dict(freq=None), dict(pos=None), dict(pos_b=-1)):
        assert call(**kw) == BAD, kw
    assert call(head_dim=1026) == UNSUP
    assert call(head_dim=1024, rot_dim=514) == UNSUP
    assert call(batch=1 << 20, tokens=1 << 20) == SHAPE
    assert call(freq=A + 4) == ALIGN and call(pos=A + 2) == ALIGN
    assert call(qi=heads(A + 1, H, N, D)) == ALIGN
    assert call(qi=Heads(A, H, -1, D, D)) == BAD                    # a negative stride
    assert call(qo=Heads(A + MB, 3, 3 * N * D, N * D, D)) == SHAPE  # head counts differ
    assert call(qo=Heads(A + MB, H, H * N * D, N * D, 0)) == BAD    # an output that repeats itself
    assert call(qo=Heads(A + MB, H, H * N * D, D, D)) == BAD        # heads and tokens overlap
    assert call(qo=heads(A + 64, H, N, D)) == BAD                   # overlaps its input without being it
    assert call(ko=heads(A + MB, 2, N, D)) == BAD                   # Q's and K's outputs are one
    assert call(qo=heads(A + 2 * MB, H, N, D)) == BAD               # Q's output is K's input
    assert call(qi=Heads(A, H, 1 << 62, N * D, D)) == SHAPE         # offsets past 64 bits
    assert call(qi=Heads(A, 1 << 30, 0, 0, D), qo=Heads(A + MB, 1 << 30, 1 << 50, 1 << 12, D)) in (SHAPE, BAD)
    assert lib.sva_rotary(RotaryParams(**good), A, A, N, heads(A, H, N, D), heads(A + MB, H, N, D), heads(A, 2, N, D),
                          None, None) == BAD                        # K without its output
    assert lib.sva_rotary(None, A, A, N, None, None, None, None, None) == BAD


def a_cache(fmt=1, pages=4, kv=2, page=64, d=64, at=A, scale=A + MB):
    return Cache(fmt, pages, kv, page, d, at, at + 2 * MB, scale, scale)


def test_cache_refusals(lib):
    B, N, D = 2, 5, 64
    k, v = heads(A + 4 * MB, 2, N, D), heads(A + 5 * MB, 2, N, D)

    def write(c=None, batch=B, tokens=N, dtype=0, k=k, v=v, slots=A, sb=N):
        return lib.sva_cache_write(c or a_cache(), batch, tokens, dtype, k, v, slots, sb, None)

    def read(c=None, batch=B, tokens=N, dtype=0, k=k, v=v, slots=A, sb=N):
        return lib.sva_cache_read(c or a_cache(), batch, tokens, dtype, slots, sb, k, v, None)

    for f in (write, read):
        for kw in (dict(c=a_cache(fmt=3)), dict(c=a_cache(pages=0)), dict(c=a_cache(kv=0)), dict(c=Cache(1, 4, 2, 64, 64, None, A, A, A)),
                   dict(c=Cache(1, 4, 2, 64, 64, A, A + MB, None, A)), dict(batch=0), dict(tokens=0), dict(dtype=2),
                   dict(slots=None), dict(sb=-1), dict(k=Heads(None, 2, 0, 0, 0)), dict(v=Heads(A, 2, -1, 64, 64))):
            assert f(**kw) == BAD, kw
        for kw in (dict(c=a_cache(page=48)), dict(c=a_cache(page=8)), dict(c=a_cache(page=512)), dict(c=a_cache(d=96))):
            assert f(**kw) == UNSUP, kw
        for kw in (dict(c=a_cache(pages=1 << 26)), dict(batch=1 << 16, tokens=1 << 16), dict(k=heads(A, 3, N, D))):
            assert f(**kw) == SHAPE, kw
        for kw in (dict(c=a_cache(at=A + 8)), dict(c=a_cache(scale=A + 4)), dict(slots=A + 2),
                   dict(k=heads(A + 8, 2, N, D)), dict(v=Heads(A, 2, 2 * N * D, N * D + 4, D))):
            assert f(**kw) == ALIGN, kw
    # outputs of the read must not repeat themselves or be one
    assert read(k=Heads(A + 4 * MB, 2, 2 * N * D, 0, D)) == BAD
    assert read(k=v, v=v) == BAD
    assert lib.sva_cache_write(None, B, N, 0, k, v, A, N, None) == BAD


def test_cache_attention_refusals(lib):
    B, H, T, D = 2, 4, 3, 64
    q, o = heads(A + 4 * MB, H, T, D), heads(A + 5 * MB, H, T, D)
    k, v = heads(A + 6 * MB, 2, T, D), heads(A + 7 * MB, 2, T, D)
    good = dict(batch=B, heads=H, queries=T, max_pages=32, softmax_scale=0.0, out_dtype=0)
    need = ctypes.c_size_t()
    assert lib.sva_cache_attention_workspace(a_cache(), CacheQuery(**good), need) == OK and need.value > 0
    W = need.value

    def call(c=None, q=q, table=A, lens=A, k=k, v=v, mask=A, mb=T * T, counts=A, ws=A + 8 * MB, wb=W, out=o, lse=A, **kw):
        return lib.sva_cache_attention(c or a_cache(), CacheQuery(**{**good, **kw}), q, table, lens, k, v, mask, mb, counts,
                                       ws, wb, out, lse, None)

    for kw in (dict(batch=0), dict(heads=0), dict(queries=0), dict(max_pages=0), dict(out_dtype=2),
               dict(softmax_scale=math.nan), dict(softmax_scale=math.inf), dict(table=None), dict(lens=None), dict(v=None),
               dict(mb=-1), dict(q=None), dict(out=None), dict(ws=None), dict(c=a_cache(fmt=7)),
               dict(out=q), dict(out=Heads(A + 5 * MB, H, H * T * D, 0, D))):
        assert call(**kw) == BAD, kw
    for kw in (dict(heads=3), dict(max_pages=1 << 26), dict(wb=W - 1), dict(batch=65537), dict(q=heads(A, 2, T, D)),
               dict(k=heads(A, 4, T, D)), dict(out=heads(A + 5 * MB, 2, T, D))):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(table=A + 2), dict(lens=A + 1), dict(counts=A + 2), dict(lse=A + 2), dict(ws=A + 8 * MB + 128),
               dict(q=heads(A + 4 * MB + 8, H, T, D)), dict(out=Heads(A + 5 * MB, H, H * T * D + 4, T * D, D)),
               dict(k=heads(A + 2, 2, T, D))):
        assert call(**kw) == ALIGN, kw
    assert call(queries=1025) == UNSUP
    assert call(c=a_cache(d=80)) == UNSUP
    # the bound on the workspace that the header gives, over shapes
    for d in (64, 112, 128):
        for t in (1, 2, 8, 33, 64, 1024):
            for h in (2, 16, 128):
                qry = CacheQuery(**{**good, "queries": t, "heads": h, "max_pages": 4096, "batch": 64})
                assert lib.sva_cache_attention_workspace(a_cache(d=d), qry, need) == OK
                assert 0 < need.value <= 66 * 2 ** 20
    one = CacheQuery(**{**good, "max_pages": 1, "queries": 1})       # a short cache is not divided
    assert lib.sva_cache_attention_workspace(a_cache(), one, need) == OK and need.value == 0
    assert lib.sva_cache_attention_workspace(a_cache(), one, None) == BAD


def test_binding_refuses_host_tensors_and_wrong_names():
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    plan = {"head_dim": 64, "rot_dim": 64, "layout": "half", "magnitude": 1.0, "freq": torch.zeros(32, dtype=torch.float64)}
    pos = torch.zeros((1, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        sva.rotary(plan, pos, x)
    with pytest.raises(TypeError):
        sva.rotary(plan, pos, x.to(torch.float16))
    with pytest.raises(ValueError, match="channels"):
        sva.rotary(plan, pos, x[..., :32])
    with pytest.raises(ValueError):
        sva.rotary(plan, pos, x[0])
    with pytest.raises(ValueError, match="layout"):
        sva.rotary_plan(64, layout="quarter", device="cpu")
    with pytest.raises(ValueError, match="scaling"):
        sva.rotary_plan(64, scaling="cubic", device="cpu")
    with pytest.raises(ValueError, match="exceeds"):
        sva.rotary_plan(64, rot_dim=66, device="cpu")
    with pytest.raises(sva.SvaError):
        sva.rotary_plan(64, rot_dim=31, device="cpu")
    assert sva.rotary_plan(64, rot_dim=32, device="cpu")["freq"].dtype == torch.float64
    with pytest.raises(ValueError, match="fmt"):
        sva.kv_cache(1, 1, 64, fmt="int4", device="cpu")
    cache = sva.kv_cache(2, 2, 64, 16, fmt="int8", device="cpu")
    assert cache["k"].shape == (2, 2, 16, 64) and cache["k"].dtype == torch.int8
    assert cache["k_scale"].shape == (2, 2, 16) and sva.kv_cache(1, 1, 64, fmt="bf16", device="cpu")["k_scale"] is None
    for f in (lambda: sva.cache_write(cache, x, x, pos), lambda: sva.cache_read(cache, pos),
              lambda: sva.cache_attention(cache, x, pos, pos[:, 0])):
        with pytest.raises(ValueError, match="device tensor"):
            f()
