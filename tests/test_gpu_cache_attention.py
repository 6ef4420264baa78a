"""sva_cache_attention on the GPU against oracle/kv_cache.py: formats, head groups,
page sizes, lengths from none to many workgroups, trees, empty rows, what lies in
masked places, strides, graphs and streams."""
import itertools

import numpy as np
import pytest

import paper_2606_23743_amd as sva

from .cache_cases import attend, bf16_normal, check, host_cache, to_gpu
from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def trees(g, B, T):
    m = np.zeros((B, T, T), np.uint8)
    for b in range(B):
        for t in range(T):
            if t:
                m[b, t] = m[b, g.integers(0, t)]
            m[b, t, t] = 1
    return m


class Case:
    """Host and device inputs of one call."""

    def __init__(self, seed, B, kv, G, T, D, page, fmt, lengths, drafts=True, scale=1.0, spare=2, token_major=True):
        g = self.g = np.random.default_rng(seed)
        self.B, self.kv, self.T, self.D, self.page = B, kv, T, D, page
        self.lengths = np.array(lengths)
        P = max(1, -(-int(max(lengths)) // page))
        pages = B * P + spare
        self.host, self.values = host_cache(g, pages, kv, page, D, fmt, scale)
        self.table = g.permutation(pages)[:B * P].reshape(B, P).astype(np.int32)
        mk = lambda h, s=1.0: bf16_normal(g, (B, T, h, D), s).transpose(1, 2) if token_major else bf16_normal(g, (B, h, T, D), s)  # noqa: E731
        self.q = mk(kv * G, 1.5)
        self.k_new, self.v_new = (mk(kv), mk(kv)) if drafts else (None, None)
        say(f"[cache attention] B={B} kv={kv} G={G} T={T} D={D} page={page} {fmt} lengths={list(lengths)[:6]} drafts={drafts}")

    def call(self, mask=None, counts=None, **kw):
        dev = lambda x: None if x is None else x.cuda()  # noqa: E731
        return sva.cache_attention(to_gpu(self.host), self.q.cuda(), i32(self.table), i32(self.lengths), dev(self.k_new),
                                   dev(self.v_new), mask=None if mask is None else torch.from_numpy(mask).cuda(),
                                   counts=None if counts is None else i32(counts), want_lse=True, **kw)

    def want(self, mask=None, counts=None, scale=None):
        return attend(self.values, self.q, self.table, self.lengths, self.page, self.k_new, self.v_new, mask, counts, scale)

    def keys(self):
        return int(max(self.lengths)) + self.T

    def run(self, mask=None, counts=None, f32=False, rows=None, scale=None):
        out, lse = self.call(mask, counts, out_dtype="f32" if f32 else "bf16", softmax_scale=scale or 0.0)
        torch.cuda.synchronize()
        worst = check(out, lse, self.want(mask, counts, scale), self.keys(), self.D, f32, rows)
        say(f"   worst error / bound: {worst:.3f}")
        return out, lse


@pytest.mark.parametrize("fmt,D,f32", itertools.product(["bf16", "e4m3", "int8"], [64, 112, 128], [False, True]))
def test_one_token(fmt, D, f32):
    Case(1, 4, 2, 4, 1, D, 16, fmt, [0, 1, 33, 300]).run(f32=f32)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_lengths_around_steps_and_pages(page, fmt):
    n = [0, 1, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 640, 700]
    Case(page, len(n), 1, 2, 1, 64, page, fmt, n, drafts=False).run()


@pytest.mark.parametrize("G,T", [(1, 1), (16, 1), (17, 1), (8, 3), (3, 11), (1, 64), (5, 13), (8, 16), (6, 48), (1, 130), (3, 129)])
@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("int8", 112), ("bf16", 64)])
def test_row_tiles_and_trees(G, T, fmt, D):
    c = Case(G * 100 + T, 2, 2, G, T, D, 32, fmt, [45, 290])
    c.run(mask=trees(c.g, 2, T))


@pytest.mark.parametrize("G,T", [(16, 2), (33, 1), (12, 4), (7, 7), (49, 1), (64, 1), (64, 2), (129, 1), (64, 4), (257, 1), (1, 257)])
@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_rows_on_both_sides_of_each_form(G, T, fmt):
    c = Case(G + T, 2, 1, G, T, 64, 64, fmt, [1100, 70])
    counts = np.array([T, max(1, T - 1)])
    rows = np.broadcast_to(np.arange(T)[None, None] < counts[:, None, None], (2, G, T))
    c.run(mask=trees(c.g, 2, T), counts=counts, rows=rows)


@pytest.mark.parametrize("page", [16, 64, 128, 256])
@pytest.mark.parametrize("fmt,D,G,T", [("bf16", 128, 4, 20), ("e4m3", 112, 2, 100), ("int8", 64, 3, 40), ("int8", 128, 1, 130)])
def test_many_rows_lengths_around_tiles_and_bad_pages(page, fmt, D, G, T):
    n = [0, 1, 63, 64, 65, 129, 700, 1000]
    c = Case(page + T, len(n), 1, G, T, D, page, fmt, n)
    c.table[5, 0] = -1
    c.table[6, -1 if page > 64 else 3] = c.values["k"].shape[0] + 5
    c.run(mask=trees(c.g, len(n), T))


@pytest.mark.parametrize("fmt,D,T", itertools.product(["bf16", "e4m3", "int8"], [64, 112, 128], [9, 40]))
def test_float32_result(fmt, D, T):
    c = Case(T, 2, 1, 2, T, D, 64, fmt, [200, 77])
    c.run(f32=True, mask=trees(c.g, 2, T))


def test_causal_and_custom_scale():
    Case(5, 3, 2, 2, 21, 128, 64, "e4m3", [100, 0, 31]).run(scale=0.31)


def test_shared_mask_and_bool_and_head_major():
    c = Case(6, 3, 2, 2, 9, 64, 16, "int8", [40, 80, 3], token_major=False)
    m = trees(c.g, 1, 9)[0]
    out, lse = c.run(mask=m)
    out2, _ = c.call(m.astype(bool))
    assert torch.equal(out, out2)


def test_empty_rows_give_zeros():
    c = Case(7, 3, 2, 3, 6, 64, 16, "e4m3", [0, 20, 0])
    m = trees(c.g, 3, 6)
    m[0, 2] = 0
    m[2] = 0
    m[1, 4] = 0
    out, lse = c.run(mask=m)
    assert bool((out[2] == 0).all()) and bool(torch.isneginf(lse[2]).all())
    assert bool((out[0, :, 2] == 0).all()) and bool(torch.isneginf(lse[0, :, 2]).all())
    assert bool(torch.isfinite(lse[1]).all())


@pytest.mark.parametrize("T", [1, 5, 40])
def test_counts_leave_other_rows(T):
    c = Case(8 + T, 5, 2, 4, T, 128, 32, "int8", [64, 33, 0, 10, 500])
    counts = np.array([T, 0, max(1, T // 2), T + 9, -3])
    out = torch.full((5, 8, T, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((5, 8, T), 7.0, device="cuda")
    m = trees(c.g, 5, T)
    c.call(m, counts, out=out, lse=lse)
    torch.cuda.synchronize()
    rows = np.broadcast_to(np.arange(T)[None, None] < counts[:, None, None], (5, 8, T))
    check(out, lse, c.want(m, counts), c.keys(), 128, rows=rows)
    off = torch.from_numpy(~rows).cuda()
    assert bool((out[off] == 7).all()) and bool((lse[off] == 7).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_what_lies_behind_a_length_or_on_a_bad_page_does_not_matter(fmt):
    c = Case(9, 3, 2, 2, 3, 64, 16, fmt, [37, 5, 64])
    c.table[2, 1] = -1
    c.table[0, 0] = len(c.host["k"]) + 5
    want = c.want()
    live = np.zeros(c.host["k"].shape[:3], bool)
    for b in range(3):
        for j in range(c.lengths[b]):
            p = c.table[b, j // 16]
            if 0 <= p < len(live):
                live[p, :, j % 16] = True
    dead = torch.from_numpy(~live)
    for n in ("k", "v"):                                  # NaN codes, NaN and Inf scales
        c.host[n][dead] = {"bf16": float("nan"), "e4m3": 0x7F, "int8": -128}[fmt]
        if fmt != "bf16":
            c.host[n + "_scale"][dead] = float("nan") if n == "k" else float("inf")
    out, lse = c.call()
    torch.cuda.synchronize()
    check(out, lse, want, c.keys(), 64)


@pytest.mark.parametrize("f32,T", [(False, 7), (True, 7), (False, 70)])
def test_inf_and_nan_of_masked_drafts_stay_out(f32, T):
    """A drafted token whose K and V hold Inf and NaN: rows that do not see it are as without it, rows that do
    see an Inf in V get it."""
    c = Case(10, 2, 2, 2, T, 128, 64, "e4m3", [50, 0])
    m = trees(c.g, 2, T)
    m[:, :, 3] = 0
    m[:, 3, 3] = 1
    want = c.want(m)
    for x, val in ((c.k_new, float("nan")), (c.v_new, float("inf"))):
        x[:, 0, 3, 5] = val
        x[:, 1, 3, 17] = -float("inf")
    out, lse = c.call(m, out_dtype="f32" if f32 else "bf16")
    torch.cuda.synchronize()
    rows = np.ones((2, 4, T), bool)
    rows[:, :, 3] = False
    check(out, lse, want, c.keys(), 128, f32, rows)
    # V alone: seen by row 3 with a weight above zero
    c2 = Case(10, 2, 2, 2, T, 128, 64, "e4m3", [50, 0])
    c2.v_new[:, :, 3, 5] = float("inf")
    out, _ = c2.call(m)
    assert bool(torch.isposinf(out[:, :, 3, 5]).all())
    others = torch.ones(out.shape, dtype=torch.bool, device="cuda")
    others[:, :, 3, 5] = False
    assert bool(torch.isfinite(out[others]).all())


def test_large_logits_and_growing_maximum():
    """Logits that grow along the sequence by more than float32's range of weights: the running maximum moves."""
    c = Case(11, 1, 1, 2, 1, 64, 64, "bf16", [700], drafts=False)
    ramp = np.linspace(0, 60, 700)
    for j in range(700):
        p = c.table[0, j // 64]
        c.host["k"][p, 0, j % 64] = torch.full((64,), float(ramp[j] / 8), dtype=torch.bfloat16)
        c.values["k"][p, 0, j % 64] = c.host["k"][p, 0, j % 64].double().numpy()
    c.q[:] = 1.5
    c.run(f32=True)
    c.q[:] = -1.5
    c.run(f32=True)


@pytest.mark.parametrize("fmt,kv,G,T,D", [("e4m3", 1, 4, 1, 128), ("int8", 2, 8, 5, 64), ("bf16", 1, 1, 100, 112)])
def test_one_sequence_over_all_workgroups(fmt, kv, G, T, D):
    c = Case(12, 1, kv, G, T, D, 64, fmt, [21000])
    c.run(mask=trees(c.g, 1, T))


def test_many_sequences():
    n = np.random.default_rng(13).integers(0, 90, 150)
    n[77] = 6000
    c = Case(13, 150, 2, 2, 2, 64, 32, "e4m3", n)
    c.run(mask=trees(c.g, 150, 2))


@pytest.mark.parametrize("B,kv,T", [(63, 9, 2), (64, 8, 1), (65, 1, 3), (200, 3, 1), (1025, 1, 2), (4097, 1, 1), (4200, 2, 1)])
@pytest.mark.parametrize("long", [False, True])
def test_batches_that_lanes_and_their_entries_divide(B, kv, T, long):
    """Pages shared by entries; lengths short but for a few, counts of zero among them."""
    c = Case.__new__(Case)
    g = c.g = np.random.default_rng(B + long)
    c.B, c.kv, c.T, c.D, c.page = B, kv, T, 64, 64
    c.lengths = g.integers(0, 40, B)
    if long:
        c.lengths[g.choice(B, 12, replace=False)] = g.integers(300, 2500, 12)
        c.lengths[[0, B - 1]] = 1500, 2300
    columns = 40 if long else 5
    c.host, c.values = host_cache(g, 90, kv, 64, 64, "e4m3")
    c.table = g.integers(0, 90, (B, columns)).astype(np.int32)
    c.q, c.k_new, c.v_new = bf16_normal(g, (B, 2 * kv, T, 64), 1.5), bf16_normal(g, (B, kv, T, 64)), bf16_normal(g, (B, kv, T, 64))
    say(f"[cache attention] B={B} kv={kv} T={T} long={long}")
    c.run()
    counts = g.integers(0, T + 1, B)
    counts[[0, B - 1]] = 1, T
    out, lse = c.call(counts=counts, out=torch.full((B, 2 * kv, T, 64), 7.0, dtype=torch.bfloat16, device="cuda"),
                      lse=torch.full((B, 2 * kv, T), 7.0, device="cuda"))
    torch.cuda.synchronize()
    there = np.broadcast_to((np.arange(T) < counts[:, None])[:, None], (B, 2 * kv, T))
    check(out, lse, c.want(counts=counts), c.keys(), 64, False, there)
    assert (out.float().cpu().numpy()[~there] == 7).all() and (lse.cpu().numpy()[~there] == 7).all()


def test_lengths_past_the_table_are_clamped():
    c = Case(14, 2, 1, 1, 1, 64, 16, "int8", [32, 20])
    c.lengths = np.array([99999, -5])
    c.run()


def test_same_bits_again_and_strided_output():
    c = Case(15, 3, 2, 4, 5, 128, 64, "e4m3", [3000, 17, 900])
    out, lse = c.run()
    for _ in range(3):
        again, l2 = c.call()
        assert torch.equal(out, again) and torch.equal(lse, l2)
    wide = torch.full((3, 5, 8 + 1, 128 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    view = wide[:, :, 1:, 8:].transpose(1, 2)
    c.call(out=view)
    assert torch.equal(view, out) and bool((wide[:, :, 0] == 3).all()) and bool((wide[..., :8] == 3).all())


def test_graphs_share_a_workspace_and_replay():
    c = Case(16, 2, 2, 4, 3, 128, 64, "int8", [2500, 700])
    d = Case(17, 1, 1, 8, 1, 128, 64, "bf16", [3000])
    runs = []
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    for x in (c, d):
        dev = dict(cache=to_gpu(x.host), q=x.q.cuda(), page_table=i32(x.table), lengths=i32(x.lengths),
                   k_new=x.k_new.cuda(), v_new=x.v_new.cuda(), out=torch.zeros(x.q.shape, dtype=torch.bfloat16, device="cuda"),
                   workspace=ws)
        sva.cache_attention(**dev)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sva.cache_attention(**dev)
        runs.append((x, dev, graph))
    for rep in range(4):
        for x, dev, graph in runs:
            x.lengths = np.maximum(1, x.lengths - 300 * rep)
            dev["lengths"].copy_(i32(x.lengths))
            dev["q"].copy_(bf16_normal(x.g, tuple(x.q.shape)))
            graph.replay()
        for x, dev, graph in runs:
            eager, _ = sva.cache_attention(**{**dev, "out": None, "workspace": None})
            torch.cuda.synchronize()
            assert torch.equal(eager, dev["out"]), rep


def test_side_stream():
    c = Case(18, 2, 2, 4, 3, 64, 64, "e4m3", [2500, 700])
    want, wl = c.call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        dev = to_gpu(c.host)
        args = (dev, c.q.cuda(), i32(c.table), i32(c.lengths), c.k_new.cuda(), c.v_new.cuda())
        torch.cuda.current_stream().synchronize()
        out, lse = sva.cache_attention(*args, want_lse=True, stream=side)
        junk = [torch.full((1 << 22,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(16)]
        torch.cuda.synchronize()
        del junk
        assert torch.equal(out, want) and torch.equal(lse, wl)


def test_binding_refusals():
    c = Case(19, 2, 1, 2, 3, 64, 16, "int8", [20, 5])
    dev, q, t, n, k, v = to_gpu(c.host), c.q.cuda(), i32(c.table), i32(c.lengths), c.k_new.cuda(), c.v_new.cuda()
    good = torch.ones((2, 3, 3), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="go together"):
        sva.cache_attention(dev, q, t, n, k)
    with pytest.raises(ValueError, match="without drafted"):
        sva.cache_attention(dev, q, t, n, mask=good)
    with pytest.raises(ValueError, match="shape"):
        sva.cache_attention(dev, q, t, n, k, v, mask=good[:, :2])
    with pytest.raises(ValueError, match="contiguous"):
        sva.cache_attention(dev, q, t, n, k, v, mask=good.transpose(1, 2))
    with pytest.raises(TypeError):
        sva.cache_attention(dev, q, t, n, k, v, mask=good.float())
    with pytest.raises(TypeError):
        sva.cache_attention(dev, q.float(), t, n, k, v)
    with pytest.raises(TypeError):
        sva.cache_attention(dev, q, t.long(), n, k, v)
    with pytest.raises(ValueError, match="shape"):
        sva.cache_attention(dev, q, t, n[:1], k, v)
    with pytest.raises(ValueError):
        sva.cache_attention(dev, q, t, n, k, v, counts=n[:1])
    with pytest.raises(sva.SvaError):
        sva.cache_attention(dev, q, t, n, k, v, out=q)
    long_table = torch.zeros((2, 100), dtype=torch.int32, device="cuda")     # past what is left undivided
    assert sva.cache_attention_workspace(dev, 2, 2, 3, 100) > 256
    with pytest.raises(sva.SvaError):
        sva.cache_attention(dev, q, long_table, n, k, v, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        sva.cache_attention(dev, q, long_table, n, k, v, workspace=torch.empty(1 << 26, device="cuda"))


@pytest.mark.parametrize("fmt,tol", [("bf16", 0.0), ("int8", 0.02), ("e4m3", 0.12)])
def test_a_generation_loop(fmt, tol):
    """The operators together, as a program uses them: a prompt's K rotated and written, then steps that draft a
    tree, attend over cache and drafts, and write the accepted tokens' K and V.  At the end the cache reads back
    as the accepted tokens' rotated K (within the format's rounding) and a step's attention equals attention over
    the whole sequence by the dense operator on what reads back."""
    g = np.random.default_rng(20)
    B, kv, G, D, page, rounds, T = 2, 2, 4, 128, 16, 4, 5
    H = kv * G
    prompt = 40
    total = prompt + rounds * T
    cache = sva.kv_cache(B * (-(-total // page)), kv, D, page, fmt)
    table = torch.randperm(B * (-(-total // page))).reshape(B, -1).to(torch.int32).cuda()
    plan = sva.rotary_plan(D, layout="half", scaling="yarn", factor=4.0, original_len=64)

    def project(n):
        qkv = bf16_normal(g, (B, n, H + 2 * kv, D)).cuda()       # one fused projection, taken as it lies
        return (qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + kv].transpose(1, 2), qkv[:, :, H + kv:].transpose(1, 2))

    def slots_of(pos):
        pos = pos.long()
        return (torch.gather(table, 1, (pos // page).clamp(max=table.shape[1] - 1)) * page + pos % page).to(torch.int32)

    pos = torch.arange(prompt, device="cuda", dtype=torch.int32).expand(B, prompt).contiguous()
    q, k, v = project(prompt)
    q, k = sva.rotary(plan, pos, q, k, q_out=q, k_out=k)         # in place in the projection's buffer
    sva.cache_write(cache, k, v, slots_of(pos))
    kept_k, kept_v = [[k[b].clone()] for b in range(B)], [[v[b].clone()] for b in range(B)]
    lengths = torch.full((B,), prompt, dtype=torch.int32, device="cuda")
    for r in range(rounds):
        mask = trees(g, B, T)
        depth = mask.sum(axis=2) - 1
        pos = lengths[:, None] + torch.from_numpy(depth.astype(np.int32)).cuda()
        q, k, v = project(T)
        q, k = sva.rotary(plan, pos, q, k, q_out=q, k_out=k)
        out, _ = sva.cache_attention(cache, q, table, lengths, k, v, mask=torch.from_numpy(mask).cuda())
        # accept the path to one node of each tree: its tokens, in order of depth
        slots = torch.full((B, T), -1, dtype=torch.int32, device="cuda")
        accepted = []
        for b in range(B):
            path = np.flatnonzero(mask[b, g.integers(0, T)])
            accepted.append(len(path))
            at = torch.from_numpy(path).cuda()
            slots[b, at] = slots_of(pos)[b, at]
            kept_k[b].append(k[b][:, at].clone())
            kept_v[b].append(v[b][:, at].clone())
        sva.cache_write(cache, k, v, slots)
        lengths = lengths + torch.tensor(accepted, dtype=torch.int32, device="cuda")
    n = lengths.tolist()
    for b in range(B):
        every = torch.arange(n[b], device="cuda", dtype=torch.int32)[None]
        s = (table[b:b + 1].gather(1, (every // page).long()) * page + every % page).to(torch.int32)
        rk, rv = sva.cache_read(cache, s)
        for got, want in ((rk[0], torch.cat(kept_k[b], 1)), (rv[0], torch.cat(kept_v[b], 1))):
            top = want.float().abs().amax(-1, keepdim=True)
            assert bool(((got.float() - want.float()).abs() <= tol * top).all())
        # one more token whose K and V are the last ones of the sequence: dense attention's last row
        prob = sva.problem(1, H, n[b], D, (1, 1, n[b]), 64)
        qq = bf16_normal(g, (1, H, n[b], D)).cuda()
        kk, vv = (x.repeat_interleave(G, 1).contiguous() for x in (rk, rv))
        dense, _ = sva.dense_attention(prob, qq, kk, vv)
        step, _ = sva.cache_attention(cache, qq[:, :, -1:], table[b:b + 1], lengths[b:b + 1])
        # both round weights and results to bf16; the cache's values were rounded to bf16 on reading
        err = (step[:, :, 0].float() - dense[:, :, -1].float()).abs().max()
        assert float(err) <= 3 * 2.0 ** -8 * float(vv.float().abs().max()), float(err)
