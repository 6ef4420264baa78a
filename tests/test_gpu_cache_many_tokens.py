"""Rotary positions and cache writes of 268 million tokens: more workgroups than one launch may hold."""
import pytest

import paper_2606_23743_amd as sva

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

B, N = 65537, 4097                                       # over 2^28 tokens; 16 of them make a workgroup


def test_rotary_past_one_launch():
    """One head of two channels, in place: the same bits as the last entries alone."""
    say(f"[rotary] {B * N} tokens")
    plan = sva.rotary_plan(2, layout="interleaved")
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    x = torch.empty((B, 1, N, 2), dtype=torch.bfloat16, device="cuda")
    x[..., 0], x[..., 1] = 1.0, 0.5
    want, _ = sva.rotary(plan, pos, x[:1].clone())
    sva.rotary(plan, pos, x, q_out=x)
    torch.cuda.synchronize()
    for b0 in range(0, B, 4096):                         # every entry is alike
        assert bool((x[b0:b0 + 4096] == want).all()), b0


def test_cache_write_past_one_launch():
    """Rows that repeat themselves; all but a few tokens have no slot."""
    say(f"[cache write] {B * N} tokens")
    D = 128
    g = torch.Generator(device="cuda").manual_seed(7)
    rows = torch.randn((B, 1, 1, D), generator=g, device="cuda", dtype=torch.bfloat16)
    slots = torch.full((B, N), -1, dtype=torch.int32, device="cuda")
    at = [(0, 0), (0, N - 1), (30000, 17), (B // 2, 4000), (B - 2, N - 1), (B - 1, 0), (B - 1, N - 1)]
    for i, (b, n) in enumerate(at):
        slots[b, n] = 2 * i + 1
    k = rows.expand(B, 1, N, D)
    cache, small = sva.kv_cache(1, 1, D, 16, "int8"), sva.kv_cache(1, 1, D, 16, "int8")
    sva.cache_write(cache, k, k, slots)
    few = rows[[b for b, _ in at], :, 0][None].transpose(1, 2).contiguous()
    sva.cache_write(small, few, few, torch.arange(1, 2 * len(at), 2, dtype=torch.int32, device="cuda")[None])
    torch.cuda.synchronize()
    for n in cache:
        assert torch.equal(cache[n], small[n]), n
    assert int((cache["k_scale"] != 0).sum()) == len(at)
