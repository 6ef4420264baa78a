"""Layer norm, rotary positions on several axes and cross attention as a denoiser's layer
uses them: forward and back through all of them, eager, captured and replayed, and beside
the framework's other operators."""
import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import cross_attention as oca
from oracle import layer_norm as oln
from oracle import rotary_axes as oaxes

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

B, H, KV, D, N, M, C = 2, 4, 2, 64, 150, 45, 256
SECTIONS = (8, 12, 12)


def _inputs(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale)  # noqa: E731
    bf = lambda t: t.to(torch.bfloat16)  # noqa: E731
    mask = torch.rand((B, M), generator=g, device="cuda") < 0.7
    mask[:, 0] = True
    return {"x": bf(r(B, N, C)), "mod": r(B, 2 * C, scale=0.2), "wq": bf(r(H * D, C, scale=C ** -0.5)),
            "k": bf(r(B, M, KV, D)).transpose(1, 2), "v": bf(r(B, M, KV, D)).transpose(1, 2),
            "pos": r(B, N, 3, scale=9.0), "mask": mask, "go": bf(r(B, N, H, D)).transpose(1, 2)}


def _layer(t, plan):
    """Forward, then the gradients of x, of the modulation and of the encoder's states."""
    scale, shift = t["mod"][:, :C], t["mod"][:, C:]
    y, mean, rstd = sva.layer_norm(t["x"], scale, shift, unit_offset=True, want_stats=True)
    q = torch.matmul(y, t["wq"].t()).view(B, N, H, D).transpose(1, 2)
    qr, _ = sva.rotary_axes(plan, t["pos"], q)
    out, lse = sva.cross_attention(qr, t["k"], t["v"], mask=t["mask"], want_lse=True)
    dqr, dk, dv = sva.cross_attention_backward(t["go"], qr, t["k"], t["v"], out, lse, mask=t["mask"])
    dq, _ = sva.rotary_axes(plan, t["pos"], dqr, backward=True)
    dy = torch.matmul(dq.transpose(1, 2).reshape(B, N, H * D), t["wq"])
    dx, dscale, dshift = sva.layer_norm_backward(dy, t["x"], mean, rstd, scale, unit_offset=True)
    return out, lse, dx, dscale, dshift, dk, dv


def _exact(t):
    c = {n: v.double().cpu().numpy() for n, v in t.items()}
    f, axis, m = oaxes.ladders(SECTIONS)
    scale, shift = c["mod"][:, :C], c["mod"][:, C:]
    y, mean, rstd = oln.forward(c["x"], scale, shift, 1e-5, 1.0)
    q = (y @ c["wq"].T).reshape(B, N, H, D).transpose(0, 2, 1, 3)
    qr = oaxes.apply(q, c["pos"], f, axis, m, "half")
    seen = oca.seen_keys(B, M, None, c["mask"])
    out, lse = oca.forward(qr, c["k"], c["v"], seen, D ** -0.5)
    dqr, dk, dv = oca.backward(c["go"], qr, c["k"], c["v"], out, lse, seen, D ** -0.5)
    dq = oaxes.apply(dqr, c["pos"], f, axis, m, "half", True)
    dy = dq.transpose(0, 2, 1, 3).reshape(B, N, H * D) @ c["wq"]
    return out, lse, *oln.backward(dy, c["x"], mean, rstd, scale, 1.0, True), dk, dv


def test_a_layers_forward_and_gradients():
    """In the 2-norm: the norm's, the projection's, the turn's and the attention's results are rounded to
    bf16, weights and dS once more, and as many gradients on the way back: at most twelve roundings of 2^-8 on
    any path, none of which a stage enlarges here (logits of size one: an error of a logit is at most as large
    relative to its weight)."""
    t = _inputs(1)
    got = _layer(t, sva.rotary_axes_plan(D, SECTIONS))
    for name, a, w in zip(("out", "lse", "dx", "dscale", "dshift", "dk", "dv"), got, _exact(t)):
        off = np.linalg.norm(a.double().cpu().numpy() - w) / np.linalg.norm(w)
        say(f"[layer] {name}: {off:.2e}")
        assert off <= 12 * 2.0 ** -8, name


def test_captured_and_replayed():
    """A graph of the whole layer, replayed on other inputs with eager work between; two graphs."""
    plan = sva.rotary_axes_plan(D, SECTIONS)
    still = _inputs(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(still, plan)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = _layer(still, plan)
        graphs.append((g, outs))
    for seed in (3, 4, 5):
        new = _inputs(seed)
        want = [o.clone() for o in _layer(new, plan)]
        for n in still:
            still[n].copy_(new[n])
        for g, outs in graphs:
            for o in outs:
                o.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)


def test_pruned_tokens_keep_their_positions():
    """Tokens kept by the pruning turn by the places they had: gather, then rotary_axes with gathered positions."""
    T, Hh, W = 4, 10, 10
    n = T * Hh * W
    x = torch.randn((1, n, 2 * 128), device="cuda").to(torch.bfloat16)
    _, idx, _ = sva.token_select(x, 0.5)
    at = torch.arange(n, device="cuda")
    grid = torch.stack((at // (Hh * W), at // W % Hh, at % W), dim=-1).to(torch.int32)
    plan = sva.rotary_axes_plan(128, (22, 21, 21), "interleaved")
    full, _ = sva.rotary_axes(plan, grid, x.view(1, n, 2, 128).transpose(1, 2))
    kept = sva.token_gather(x, idx)
    got, _ = sva.rotary_axes(plan, grid[idx.long()], kept.view(1, -1, 2, 128).transpose(1, 2))
    assert torch.equal(got, full[:, :, idx[0].long()])


def test_one_token_after_the_other_is_the_whole_sequence():
    """Single-token steps and one call for all tokens differ by the roundings of their parts alone."""
    g = torch.Generator(device="cuda").manual_seed(9)
    q = torch.randn((2, 8, 12, 128), generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((2, 2, 3000, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    lengths = torch.tensor([3000, 1234], dtype=torch.int32, device="cuda")
    whole, lse = sva.cross_attention(q, k, v, lengths=lengths, want_lse=True)
    for n in range(12):
        one, l = sva.cross_attention(q[:, :, n:n + 1], k, v, lengths=lengths, want_lse=True)
        # weights rounded against another reference, and the result: two bf16 steps of what they weigh
        lim = 4 * 2.0 ** -8 * float(v.float().abs().mean()) + 2.0 ** -7 * whole[:, :, n:n + 1].float().abs()
        assert ((one.float() - whole[:, :, n:n + 1].float()).abs() <= lim).all()
        assert (l - lse[:, :, n:n + 1]).abs().max() <= 1e-5
