"""Calls on a side stream right after the current stream freed memory that its own
kernels, still waiting, go on to read and write: neither's results may change.  (Which
stream the memory belongs to is tested on the CPU.)"""
import numpy as np
import pytest

import paper_2606_23743_amd as sva

from .cache_cases import bf16_normal, host_cache, to_gpu
from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _calls():
    """name -> call(stream) of what allocates outputs and workspaces, on fixed inputs."""
    g = np.random.default_rng(31)
    B, kv, G, T, D, page = 2, 2, 4, 5, 128, 64
    host, _ = host_cache(g, 64, kv, page, D, "e4m3")
    cache = to_gpu(host)
    table = torch.arange(64, dtype=torch.int32, device="cuda").reshape(B, 32)
    lengths = torch.tensor([2000, 700], dtype=torch.int32, device="cuda")
    q, k, v = (bf16_normal(g, (B, h, T, D)).cuda() for h in (kv * G, kv, kv))
    rq, rk = bf16_normal(g, (B, 8, 600, D)).cuda(), bf16_normal(g, (B, 2, 600, D)).cuda()
    plan, pos = sva.rotary_plan(D), torch.arange(600, dtype=torch.int32, device="cuda")
    slots = torch.randperm(64 * page, device="cuda")[:2 * 900].reshape(2, 900).to(torch.int32)
    x = bf16_normal(g, (2, 3000, 256)).cuda()
    prob = sva.problem(1, 4, 1024, D, (1, 32, 32), 64)
    dq = [bf16_normal(g, (1, 4, 1024, D)).cuda() for _ in range(3)]
    return {
        "cache_attention": lambda s: sva.cache_attention(cache, q, table, lengths, k, v, want_lse=True, stream=s),
        "rotary": lambda s: sva.rotary(plan, pos, rq, rk, stream=s),
        "cache_read": lambda s: sva.cache_read(cache, slots, stream=s),
        "token_select": lambda s: sva.token_select(x, 0.5, stream=s),
        "dense_attention": lambda s: sva.dense_attention(prob, *dq, want_lse=True, stream=s),
    }


@pytest.mark.parametrize("name", ["cache_attention", "rotary", "cache_read", "token_select", "dense_attention"])
def test_memory_freed_under_pending_work_is_not_taken(name):
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    say(f"[side allocation] {name}")
    sizes = [t.numel() * t.element_size() for t in want] + [1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24, 1 << 26]
    for _ in range(3):
        torch.cuda.empty_cache()
        side.wait_stream(torch.cuda.current_stream())        # the inputs are there
        blocks = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes]
        sums = [torch.zeros((), dtype=torch.int64, device="cuda") for _ in sizes]
        torch.cuda._sleep(20_000_000)                        # holds the current stream back (bounded spin)
        for b, n in zip(blocks, sums):
            n.copy_((b != 0x5A).any())                       # reads them later
            b.fill_(0x33)                                    # and writes them
        del blocks, b                                        # freed under the work that waits
        got = call(side)
        torch.cuda.synchronize()
        assert all(int(n) == 0 for n in sums)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_outputs_freed_under_pending_use_are_not_taken():
    """An output that the current stream still has to read is dropped; the next call on the side stream must
    not be given its memory."""
    call = _calls()["cache_read"]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kept = []
    for _ in range(4):
        got = call(side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(5_000_000)
        kept.append([t.clone() for t in got])                # reads them after the spin
        del got
        with torch.cuda.stream(side):                        # what the side stream allocates next, it overwrites
            junk = [torch.full_like(t, 7.0) for t in want]
            del junk
    torch.cuda.synchronize()
    for got in kept:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", ["cache_attention", "rotary", "cache_read", "token_select"])
def test_a_side_stream_forked_into_a_capture(name):
    """Outputs and workspaces allocated on a side stream that takes part in a capture stay the graph's: replays, with
    eager work between them that allocates, give the eager results."""
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    say(f"[side allocation] captured {name}")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        again = call(side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        for t in (*got, *again):
            t.zero_()
        junk = [torch.full((1 << n,), 0x7F, dtype=torch.uint8, device="cuda") for n in range(16, 27)]
        eager = call(side)
        torch.cuda.synchronize()
        graph.replay()
        for n in junk:
            n.fill_(0x55)
        torch.cuda.synchronize()
        del junk
        for result in (got, again, eager):
            assert all(torch.equal(a, b) for a, b in zip(result, want))
