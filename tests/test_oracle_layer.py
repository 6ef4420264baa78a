"""Pins of the oracles of layer norm, rotary positions on several axes and cross
attention: automatic differentiation and library routines in float64, central
differences, closed forms."""
import math

import numpy as np
import pytest

from oracle import cross_attention as oca
from oracle import layer_norm as oln
from oracle import qknorm_rope, rotary, rotary_axes

pytestmark = pytest.mark.cpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("per_entry,unit", [(False, 0.0), (True, 1.0), (True, 0.0)])
def test_layer_norm_against_autograd(per_entry, unit):
    g = np.random.default_rng(1)
    B, N, C = 3, 5, 19
    x, dy = g.standard_normal((B, N, C)) * 3 + 1, g.standard_normal((B, N, C))
    w, b = (g.standard_normal((B, C) if per_entry else (C,)) for _ in range(2))
    tx, tw, tb = (torch.tensor(t, requires_grad=True) for t in (x, w, b))
    grow = (lambda t: t[:, None]) if per_entry else (lambda t: t)
    y = torch.nn.functional.layer_norm(tx, (C,), eps=1e-3) * (grow(tw) + unit) + grow(tb)
    y.backward(torch.tensor(dy))
    got, mean, rstd = oln.forward(x, w, b, 1e-3, unit)
    dx, dw, db = oln.backward(dy, x, mean, rstd, w, unit, per_entry)
    for a, t in ((got, y.detach()), (dx, tx.grad), (dw, tw.grad), (db, tb.grad)):
        assert np.allclose(a, t.numpy(), rtol=1e-11, atol=1e-11)


def test_layer_norm_of_one_channel_and_of_equal_ones():
    y, mean, rstd = oln.forward(np.full((1, 2, 1), 7.0), None, np.array([3.0]), 1e-2)
    assert np.array_equal(y, np.full((1, 2, 1), 3.0)) and np.allclose(rstd, 10.0) and np.all(mean == 7.0)
    y, _, _ = oln.forward(np.full((1, 1, 8), -2.0))
    assert np.all(y == 0.0)


def test_axes_of_a_grid_are_the_fused_producers():
    D, grid = 112, (3, 4, 5)
    sections = qknorm_rope.rope_pair_groups(D)
    f, axis, m = rotary_axes.ladders(sections)
    t, y, x = np.meshgrid(*(np.arange(n) for n in grid), indexing="ij")
    pos = np.stack([t, y, x], axis=-1).reshape(1, -1, 3)
    q = np.random.default_rng(2).standard_normal((1, 2, 60, D))
    want = qknorm_rope.apply_rope(q, qknorm_rope.rope_angles(grid, D, 10000.0))
    assert m == 1.0 and np.allclose(rotary_axes.apply(q, pos, f, axis, m, "interleaved"), want, rtol=0, atol=1e-12)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_one_axis_is_plain_rotary_and_the_gradient_its_inverse(layout):
    x = np.random.default_rng(3).standard_normal((2, 2, 7, 24))
    pos = np.arange(14).reshape(2, 7)
    f, axis, m = rotary_axes.ladders([10])
    want = rotary.apply(x, pos, *rotary.frequencies(20), layout)
    got = rotary_axes.apply(x, pos[..., None], f, axis, m, layout)
    assert np.allclose(got, want, rtol=0, atol=1e-13)
    assert np.allclose(rotary_axes.apply(got, pos[..., None], f, axis, m, layout, True), x, rtol=0, atol=1e-13)


def test_an_axis_that_is_none_of_them_does_not_turn():
    x = np.random.default_rng(4).standard_normal((1, 1, 3, 8))
    f, axis, m = rotary_axes.ladders([2, 2])
    axis = np.array([0, 5, 1, -1])
    got = rotary_axes.apply(x, np.full((1, 3, 2), 9), f, axis, m, "half")
    assert np.array_equal(got[..., [1, 3, 5, 7]], x[..., [1, 3, 5, 7]]) and not np.allclose(got[..., 0], x[..., 0])


@pytest.mark.parametrize("hide", ["none", "lengths", "mask"])
def test_cross_attention_against_autograd(hide):
    g = np.random.default_rng(5)
    B, H, kv, N, M, D = 3, 4, 2, 5, 7, 6
    q, k, v, go = (g.standard_normal(s) for s in ((B, H, N, D), (B, kv, M, D), (B, kv, M, D), (B, H, N, D)))
    lengths = np.array([7, 3, 1]) if hide == "lengths" else None
    mask = g.random((B, M)) < 0.5 if hide == "mask" else None
    if mask is not None:
        mask[:, 0] = True
    seen = oca.seen_keys(B, M, lengths, mask)
    c = 0.7
    tq, tk, tv = (torch.tensor(t, requires_grad=True) for t in (q, k, v))
    s = c * tq @ tk.repeat_interleave(H // kv, 1).transpose(2, 3)
    s = s.masked_fill(~torch.tensor(seen)[:, None, None], -math.inf)
    o = torch.softmax(s, -1) @ tv.repeat_interleave(H // kv, 1)
    o.backward(torch.tensor(go))
    out, lse = oca.forward(q, k, v, seen, c)
    assert np.allclose(out, o.detach().numpy(), atol=1e-12) and np.allclose(lse, torch.logsumexp(s, -1).detach().numpy())
    for a, t in zip(oca.backward(go, q, k, v, out, lse, seen, c), (tq, tk, tv)):
        assert np.allclose(a, t.grad.numpy(), atol=1e-12)


def test_cross_attention_gradient_against_differences():
    g = np.random.default_rng(6)
    q, k, v, go = (g.standard_normal(s) for s in ((1, 2, 3, 4), (1, 1, 5, 4), (1, 1, 5, 4), (1, 2, 3, 4)))
    seen = np.array([[True, True, False, True, True]])
    out, lse = oca.forward(q, k, v, seen, 0.5)
    grads = oca.backward(go, q, k, v, out, lse, seen, 0.5)
    h = 1e-5
    for x, dx in zip((q, k, v), grads):
        for at in list(np.ndindex(*x.shape))[::3]:
            keep = x[at]
            x[at] = keep + h
            up = (oca.forward(q, k, v, seen, 0.5)[0] * go).sum()
            x[at] = keep - h
            down = (oca.forward(q, k, v, seen, 0.5)[0] * go).sum()
            x[at] = keep
            assert abs((up - down) / (2 * h) - dx[at]) < 1e-8


def test_cross_attention_without_keys_and_with_hidden_values():
    q, k = np.ones((2, 1, 2, 4)), np.full((2, 1, 3, 4), np.nan)
    v = np.full((2, 1, 3, 4), np.inf)
    k[0, 0, 1], v[0, 0, 1] = 1.0, 5.0
    seen = oca.seen_keys(2, 3, None, np.array([[0, 1, 0], [0, 0, 0]]))
    out, lse = oca.forward(q, k, v, seen, 0.5)
    assert np.all(out[0] == 5.0) and np.all(lse[0] == 2.0) and np.all(out[1] == 0.0) and np.all(lse[1] == -np.inf)
    for d in oca.backward(np.ones_like(q), q, k, v, out, lse, seen, 0.5):
        assert np.all(d[1] == 0.0) and np.all(np.isfinite(d))
