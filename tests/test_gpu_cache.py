"""sva_cache_write and sva_cache_read on the GPU against oracle/kv_cache.py: codes and
scales equal, values rounded once; formats, types, strides, pages, odd slots."""
import itertools

import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import kv_cache as okv

from .cache_cases import CODES, bf16_normal, host_cache, to_gpu
from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _rows(g, B, kv, N, D, dtype):
    """Rows of many sizes: ordinary ones, zero rows, rows with one large channel, tiny and huge ones."""
    x = g.standard_normal((B, kv, N, D)) * np.exp(g.uniform(-6, 6, (B, kv, N, 1)))
    kind = g.integers(0, 12, (B, kv, N))
    x[kind == 0] = 0.0
    x[kind == 1, 0] *= 100.0
    x[kind == 2] *= 1e-30
    x[kind == 3] *= 1e30
    x[kind == 4] = np.round(x[kind == 4] * 4) / 4          # ties
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t


def _layout(x, token_major, pad=0):
    if token_major:
        B, H, N, D = x.shape
        y = torch.empty((B, N, H + pad, D), dtype=x.dtype, device="cuda")[:, :, pad:].transpose(1, 2)
        return y.copy_(x)
    return x.cuda()


@pytest.mark.parametrize("fmt,dtype,D", itertools.product(["bf16", "e4m3", "int8"], ["bf16", "f32"], [64, 112, 128]))
@pytest.mark.parametrize("B,kv,N,page,token_major", [(1, 1, 1, 16, False), (3, 5, 77, 32, True), (2, 8, 130, 128, False),
                                                     (40, 2, 1, 256, True)])
def test_codes_and_scales(fmt, dtype, D, B, kv, N, page, token_major):
    g = np.random.default_rng(N * D + page)
    say(f"[cache] {fmt} {dtype} D={D} B={B} kv={kv} N={N} page={page} token_major={token_major}")
    k, v = (_rows(g, B, kv, N, D, dtype) for _ in range(2))
    pages = -(-B * N // page) + 2
    host, _ = host_cache(g, pages, kv, page, D, fmt)
    cache = to_gpu(host)
    slots = g.permutation(pages * page)[:B * N].reshape(B, N).astype(np.int32)
    drop = g.random((B, N)) < 0.2
    drop[0, 0] = False
    slots_in = np.where(drop, g.choice([-1, -7, pages * page, 2 ** 31 - 1, -2 ** 31], (B, N)), slots).astype(np.int32)
    sva.cache_write(cache, _layout(k, token_major, 2), _layout(v, token_major), torch.from_numpy(slots_in).cuda())
    torch.cuda.synchronize()
    for n, x in (("k", k), ("v", v)):
        x = x.double().numpy().transpose(0, 2, 1, 3)[~drop]          # [written, kv, D]
        at = slots[~drop]
        want = host[n].clone()
        if fmt == "bf16":
            want[at // page, :, at % page] = torch.from_numpy(x).to(torch.bfloat16)
        else:
            c, s = okv.quantise_rows(x, fmt)
            scales = host[n + "_scale"].clone()
            scales[at // page, :, at % page] = torch.from_numpy(s).float()
            assert torch.equal(cache[n + "_scale"].cpu(), scales)
            codes = torch.from_numpy(c).to(torch.int8) if fmt == "int8" else \
                torch.from_numpy(c).float().to(torch.float8_e4m3fn).view(torch.uint8)
            want[at // page, :, at % page] = codes
        got = cache[n].cpu()
        if fmt == "e4m3":                                            # -0 and 0 are one value
            got, want = (torch.where(t == 128, 0, t) for t in (got, want))
        assert torch.equal(got, want), (n, int((got != want).sum()))


@pytest.mark.parametrize("fmt,dtype,D", itertools.product(["bf16", "e4m3", "int8"], ["bf16", "f32"], [64, 112, 128]))
@pytest.mark.parametrize("B,kv,N,page", [(1, 1, 1, 16), (2, 5, 75, 64), (7, 3, 40, 16)])
def test_read_back(fmt, dtype, D, B, kv, N, page):
    g = np.random.default_rng(N + D)
    pages = 9
    host, values = host_cache(g, pages, kv, page, D, fmt)
    slots = g.integers(-3, pages * page + 3, (B, N)).astype(np.int32)   # repeated and bad ones too
    say(f"[cache read] {fmt} {dtype} D={D} B={B} kv={kv} N={N} page={page}")
    k, v = sva.cache_read(to_gpu(host), torch.from_numpy(slots).cuda(), dtype=dtype)
    # into slices of something wider
    wide = torch.full((B, N, kv + 2, 2 * D), 7.0, dtype=k.dtype, device="cuda")
    views = [wide[:, :, 1:-1, i * D:(i + 1) * D].transpose(1, 2) for i in range(2)]
    sva.cache_read(to_gpu(host), torch.from_numpy(slots).cuda(), k=views[0], v=views[1], dtype=dtype)
    torch.cuda.synchronize()
    assert k.is_contiguous() and torch.equal(views[0], k) and torch.equal(views[1], v)
    assert bool((wide[:, :, 0] == 7).all()) and bool((wide[:, :, -1] == 7).all())
    ok = (slots >= 0) & (slots < pages * page)
    at = np.where(ok, slots, 0)
    for got, n in ((k, "k"), (v, "v")):
        want = values[n][at // page, :, at % page] * ok[..., None, None]
        want = want.transpose(0, 2, 1, 3)
        # float32 product, then (bf16) a second rounding
        tol = np.abs(want) * (2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0)) if fmt != "bf16" else 0.0
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


def test_shared_input_rows_and_subnormal_scales():
    """A K broadcast over heads and entries; float32 rows so small that their int8 scale is subnormal or zero."""
    D, N = 128, 5
    x = torch.zeros((1, 1, N, D), dtype=torch.float32)
    x[0, 0, 0] = torch.linspace(-1, 1, D) * 1e-37
    x[0, 0, 1] = torch.linspace(-1, 1, D) * 3e-40
    x[0, 0, 2, 3] = 2.0 ** -149
    x[0, 0, 3] = torch.linspace(-1, 1, D) * 3e38
    x[0, 0, 4] = 1.0
    for fmt in ("int8", "e4m3"):
        cache = sva.kv_cache(1, 4, D, 16, fmt)
        y = x.cuda().expand(2, 4, N, D)
        slots = torch.arange(10, dtype=torch.int32, device="cuda").reshape(2, 5)
        sva.cache_write(cache, y, y, slots)
        torch.cuda.synchronize()
        c, s = okv.quantise_rows(x[0, 0].double().numpy(), fmt)
        for b in range(2):
            for h in range(4):
                assert np.array_equal(cache["k_scale"][0, h, 5 * b:5 * b + 5].cpu().double().numpy(), s), fmt
                k = cache["k"][0, h, 5 * b:5 * b + 5].cpu()
                k = k.double() if fmt == "int8" else k.view(torch.float8_e4m3fn).double()
                assert np.array_equal(k.numpy(), c), fmt
        assert torch.equal(cache["k"], cache["v"])


def test_slots_behind_32_bit_offsets():
    """Codes past 4 GiB of K: the last pages of a cache of 4.3 billion codes."""
    D, kv, page = 128, 8, 128
    pages = (1 << 32) // (D * kv * page) + 8
    say(f"[cache] {pages} pages, {pages * kv * page * D / 2**30:.2f} GiB of K")
    cache = {"k": torch.empty((pages, kv, page, D), dtype=torch.uint8, device="cuda"),
             "v": torch.empty((pages, kv, page, D), dtype=torch.uint8, device="cuda"),
             "k_scale": torch.empty((pages, kv, page), device="cuda"), "v_scale": torch.empty((pages, kv, page), device="cuda")}
    g = np.random.default_rng(5)
    N = 3 * page + 7
    k, v = bf16_normal(g, (1, kv, N, D)).cuda(), bf16_normal(g, (1, kv, N, D)).cuda()
    slots = torch.arange(pages * page - N, pages * page, dtype=torch.int32, device="cuda")[None]
    sva.cache_write(cache, k, v, slots)
    k2, v2 = sva.cache_read(cache, slots)
    # the same rows through a small cache at the start
    small = sva.kv_cache(8, kv, D, page, "e4m3")
    s2 = torch.arange(N, dtype=torch.int32, device="cuda")[None]
    sva.cache_write(small, k, v, s2)
    k3, v3 = sva.cache_read(small, s2)
    assert torch.equal(k2, k3) and torch.equal(v2, v3) and float((k2.float() - k.float()).abs().max()) < 0.3
    # and the attention over them
    q = bf16_normal(g, (1, 16, 2, D)).cuda()
    first = pages - (N + page - 1) // page
    lead = page * (pages - first) - N                    # the first page's slots before the rows
    q_out = []
    for c, p0 in ((cache, first), (small, 0)):
        if p0:                                           # bring both to the same slots
            all_slots = torch.arange(first * page, first * page + N, dtype=torch.int32, device="cuda")[None]
            sva.cache_write(c, k, v, all_slots)
        table = torch.arange(p0, p0 + (N + page - 1) // page, dtype=torch.int32, device="cuda")[None]
        q_out.append(sva.cache_attention(c, q, table, torch.tensor([N], dtype=torch.int32, device="cuda"))[0])
    assert lead >= 0 and torch.equal(q_out[0], q_out[1])


def test_graph_and_stream():
    """Write and read captured in a graph, replayed over changing inputs; and on a side stream."""
    g = np.random.default_rng(11)
    B, kv, N, D, page = 2, 3, 50, 112, 16
    cache = sva.kv_cache(16, kv, D, page, "int8")
    k = torch.zeros((B, kv, N, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    slots = torch.randperm(16 * page)[:B * N].reshape(B, N).to(torch.int32).cuda()
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sva.cache_write(cache, k, v, slots)
        sva.cache_read(cache, slots, k=ko, v=vo)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sva.cache_write(cache, k, v, slots)
        sva.cache_read(cache, slots, k=ko, v=vo)
    for rep in range(4):
        k.copy_(bf16_normal(g, k.shape, 1 + rep))
        v.copy_(bf16_normal(g, v.shape))
        graph.replay()
        got = ko.clone(), vo.clone()
        other = sva.kv_cache(16, kv, D, page, "int8")
        sva.cache_write(other, k, v, slots, stream=side)
        side.synchronize()
        want = sva.cache_read(other, slots)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), rep


def test_formats_cover_the_binding():
    assert set(CODES) == {"bf16", "e4m3", "int8"}
    cache = sva.kv_cache(2, 2, 64, 16, "e4m3")
    k = torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device="cuda")
    bad = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="share"):
        sva.cache_write(cache, k, k, bad)
    with pytest.raises(TypeError):
        sva.cache_write(cache, k, k, bad.long()[None].expand(2, 3))
    with pytest.raises(ValueError, match="contiguous"):
        sva.cache_write(cache, k.transpose(2, 3).contiguous().transpose(2, 3), k, bad[None].expand(2, 3))
    with pytest.raises(ValueError, match="shape"):
        sva.cache_write(cache, k, k[:, :1], bad[None].expand(2, 3))
    with pytest.raises(TypeError):
        sva.cache_write({**cache, "k": cache["k"].float()}, k, k, bad[None].expand(2, 3))
    with pytest.raises(sva.SvaError):                     # rows not at multiples of 16 bytes
        wide = torch.zeros((2, 2, 3, 68), dtype=torch.bfloat16, device="cuda")[..., 4:]
        sva.cache_write(cache, wide, wide, torch.arange(6, dtype=torch.int32, device="cuda").reshape(2, 3))
