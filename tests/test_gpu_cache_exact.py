"""sva_cache_attention on inputs whose float32 arithmetic is exact (tests/cache_exact.py): every
form of the kernels, divided and joined, with bf16 and float32 results, at every head
size and cache format; and the precision of float32 results."""
import itertools

import numpy as np
import pytest

import paper_2606_23743_amd as sva

from . import cache_exact as ce
from .cache_cases import to_gpu
from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# query heads of a cache head and drafted tokens: one, two and three row tiles a wave (up to 16, 32, 48
# rows); shared keys with one and two tiles a wave (64, 128 rows), and with two passes over the keys
FORMS = [(4, 1), (6, 5), (12, 4), (7, 8), (16, 7), (5, 33)]


def _run(c, f32):
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    say(f"[cache exact] B={c.B} kv={c.kv} G={c.G} T={c.T} D={c.D} page={c.page} {c.fmt} f32={f32} up to {c.lengths.max()}")
    out = torch.full(c.q.shape, 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    lse = torch.full(c.q.shape[:3], 7.0, device="cuda")
    sva.cache_attention(to_gpu(c.cache), c.q.cuda(), i32(c.table), i32(c.lengths), c.k_new.cuda(), c.v_new.cuda(),
                        mask=torch.from_numpy(c.mask).cuda(), counts=i32(c.counts), softmax_scale=c.scale, out=out, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def _check_whole(c):
    want = c.exact()
    gone = torch.from_numpy(~want[2]).cuda()
    for f32 in (False, True):
        out, lse = _run(c, f32)
        ce.check_whole(out, lse, want, f32)
        assert bool((out[gone] == 7).all()) and bool((lse[gone] == 7).all())


@pytest.mark.parametrize("G,T", FORMS)
@pytest.mark.parametrize("fmt,D,page", itertools.product(["bf16", "e4m3", "int8"], [64, 112, 128], [16, 64]))
def test_every_form_divided(G, T, fmt, D, page):
    """1,100 keys are nine units: each a workgroup's, joined."""
    _check_whole(ce.whole_case(G * 100 + T, 2, 2, G, T, D, page, fmt, [1100, 70]))


@pytest.mark.parametrize("G,T", FORMS)
@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("e4m3", 112), ("int8", 64)])
def test_every_form_whole(G, T, fmt, D):
    """Tables of up to six units are not divided."""
    _check_whole(ce.whole_case(G * 100 + T, 3, 2, G, T, D, 32, fmt, [500, 0, 129]))


@pytest.mark.parametrize("G,T", FORMS)
@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("int8", 112), ("bf16", 64)])
def test_one_sequence_over_all_workgroups(G, T, fmt, D):
    _check_whole(ce.whole_case(G * 100 + T, 1, 4, G, T, D, 128, fmt, [21000]))


@pytest.mark.parametrize("G,T,B", [(4, 1, 300), (6, 5, 290), (12, 4, 300), (7, 8, 270), (5, 33, 140)])
@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("int8", 112), ("bf16", 64)])
def test_joins_that_follow_the_runs(G, T, B, fmt, D):
    """More segments than workgroups, a few of them long."""
    n = np.random.default_rng(B).integers(0, 60, B)
    n[[3, B // 2, B - 1]] = 1500, 2300, 990
    _check_whole(ce.whole_case(G * 100 + T, B, 2, G, T, D, 64, fmt, n, pool=50))


@pytest.mark.parametrize("G,T", FORMS)
@pytest.mark.parametrize("fmt,D,n", itertools.product(["bf16", "e4m3", "int8"], [64, 112, 128], [[1100, 70], [300, 500]]))
def test_float32_results_keep_float32_weights(G, T, fmt, D, n):
    c = ce.fine_case(G * 100 + T, 2, 2, G, T, D, 64, fmt, n)
    want = c.exact()
    out, lse = _run(c, True)
    err = ce.norm_error(out, want)
    say(f"   error {err:.2e} of the norm, allowed {ce.FINE_NORM:.2e}")
    assert err <= ce.FINE_NORM


@pytest.mark.parametrize("causal", [True, False])
def test_more_queries_than_a_call_takes_in_parts(causal):
    """1,300 tokens over a bf16 cache: a prompt's parts attend and are written in turn; a frame's tokens, which all
    see each other, are written first and attend in parts without drafted keys."""
    g = np.random.default_rng(9)
    kv, G, D, N, most, page = 2, 3, 64, 1300, 1024, 32
    q, k = np.zeros((1, kv * G, N, D)), g.integers(-3, 4, (1, kv, N, D)).astype(np.float64)
    q[..., 0], k[..., 0] = g.integers(-1, 2, (1, kv * G, N)), g.integers(0, 2, (1, kv, N))
    v = g.integers(-8, 9, (1, kv, N, D)).astype(np.float64)
    w = np.exp2(np.einsum("bhtd,bhsd->bhts", q, np.repeat(k, G, 1))) * (np.tri(N) if causal else 1.0)
    total = w.sum(axis=-1)
    want = (w @ np.repeat(v, G, 1)) / total[..., None], np.log(total), np.ones((1, kv * G, N), bool)
    say(f"[cache exact] {N} queries in parts, causal={causal}")
    dq, dk, dv = (torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda() for x in (q, k, v))
    cache = sva.kv_cache(50, kv, D, page, "bf16")
    table = torch.randperm(50)[:-(-N // page)].to(torch.int32).cuda()[None]
    at = torch.arange(N, device="cuda")
    slots = (table[0, at // page] * page + at % page).to(torch.int32)[None]
    parts = [(a, min(a + most, N)) for a in range(0, N, most)]
    if not causal:
        sva.cache_write(cache, dk, dv, slots)
    out, lse = [], []
    for a, b in parts:
        n = torch.tensor([a if causal else N], dtype=torch.int32, device="cuda")
        new = (dk[:, :, a:b], dv[:, :, a:b]) if causal else ()
        o, l = sva.cache_attention(cache, dq[:, :, a:b], table, n, *new, softmax_scale=ce.LN2, out_dtype="f32", want_lse=True)
        if causal:
            sva.cache_write(cache, *new, slots[:, a:b])
        out.append(o)
        lse.append(l)
    torch.cuda.synchronize()
    ce.check_whole(torch.cat(out, 2), torch.cat(lse, 2), want, True)
