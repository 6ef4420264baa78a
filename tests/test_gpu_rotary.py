"""sva_rotary on the GPU against oracle/rotary.py: layouts, parts of the head,
scalings, far positions, strides and alignments, in place, gradients."""
import itertools

import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import rotary as orot

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _tol(x, y, m, bf16):
    """The angle errs by half a step of a float32 turn (2^-26 turns, 9.4e-8 rad), cosine
    and sine by 2 steps (2.4e-7) and the magnitude's product, the two products and the
    sum by a half step each: 5e-7 of m (|a| + |b|), bounded by twice the row's largest
    channel; then one rounding of the result."""
    big = np.abs(x).max(axis=-1, keepdims=True)
    return 5e-7 * m * 2 * big + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(y) + 1e-38


def _case(B, H, Hk, N, D, rot, layout, dtype, backward=False, strides="plain", positions=None, in_place=False, offset=0, **kw):
    g = np.random.default_rng(B * 1000 + N + D + rot)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    say(f"[rotary] B={B} H={H}+{Hk} N={N} D={D} rot={rot} {layout} {dtype} {strides} backward={backward} in_place={in_place} {kw}")

    def tensor(heads):
        x = torch.from_numpy(g.standard_normal((B, heads, N, D)).astype(np.float32)).to(dt)
        if strides == "plain":
            y = torch.empty(B * heads * N * D + offset, dtype=dt, device="cuda")[offset:].view(B, heads, N, D)
        elif strides == "token":
            y = torch.empty((B, N, heads, D), dtype=dt, device="cuda").transpose(1, 2)
        else:                                       # a slice of something wider, odd pitches
            y = torch.empty((N, B, heads + 1, D + 3), dtype=dt, device="cuda")[:, :, 1:, 3:].permute(1, 2, 0, 3)
        return y.copy_(x), x.double().numpy()

    q, q64 = tensor(H)
    k, k64 = tensor(Hk) if Hk else (None, None)
    pos = g.integers(0, 5000, (B, N)) if positions is None else np.broadcast_to(positions, (B, N))
    plan = sva.rotary_plan(D, rot, layout, **kw)
    f, m = orot.frequencies(rot, **kw)
    p32 = torch.from_numpy(np.ascontiguousarray(pos).astype(np.int32)).cuda()
    if in_place:
        keep = [t for t in (q, k) if t is not None]
        qo, ko = sva.rotary(plan, p32, q, k, q_out=q, k_out=k, backward=backward)
        assert qo is q and ko is k and keep
    else:
        before = q.clone()
        qo, ko = sva.rotary(plan, p32, q, k, backward=backward)
        assert torch.equal(before, q)
    torch.cuda.synchronize()
    for got, x in ((qo, q64),) + (((ko, k64),) if Hk else ()):
        y = orot.apply(x, pos, f, m, layout, backward)
        z = got.double().cpu().numpy()
        assert got.shape == x.shape and got.dtype == dt
        assert np.array_equal(z[..., rot:], x[..., rot:])           # copied, bit by bit
        assert (np.abs(z - y) <= _tol(x, y, m, dtype == "bf16")).all(), np.abs(z - y).max()


@pytest.mark.parametrize("layout,dtype", itertools.product(["half", "interleaved"], ["bf16", "f32"]))
@pytest.mark.parametrize("D,rot", [(128, 128), (112, 112), (64, 32), (128, 36), (112, 2), (66, 50), (256, 256), (1024, 512)])
def test_layouts_and_parts(layout, dtype, D, rot):
    _case(2, 3, 1, 37, D, rot, layout, dtype)


@pytest.mark.parametrize("layout,dtype,strides,in_place,backward",
                         itertools.product(["half", "interleaved"], ["bf16", "f32"], ["plain", "token", "odd"],
                                           [False, True], [False, True]))
def test_strides_in_place_backward(layout, dtype, strides, in_place, backward):
    _case(3, 4, 2, 19, 64, 48, layout, dtype, backward=backward, strides=strides, in_place=in_place)


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0, base=500000.0),
                                dict(scaling="yarn", factor=16.0, original_len=4096), dict(magnitude=0.5)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_scalings(kw, layout):
    _case(1, 5, 5, 301, 128, 64, layout, "f32", **kw)


def test_far_negative_and_shared_positions():
    far = np.array([0, 1, -1, 1 << 20, -(1 << 24), 2 ** 31 - 1, -2 ** 31, 123456789])
    for layout in ("half", "interleaved"):
        _case(2, 2, 2, 8, 128, 128, layout, "f32", positions=far)


@pytest.mark.parametrize("B,H,Hk,N", [(1, 1, 0, 1), (64, 32, 8, 1), (1, 300, 1, 3), (5, 7, 0, 257), (1, 1, 1, 4099)])
def test_sizes(B, H, Hk, N):
    _case(B, H, Hk, N, 128, 128, "half", "bf16")


@pytest.mark.parametrize("dtype,layout", itertools.product(["bf16", "f32"], ["half", "interleaved"]))
@pytest.mark.parametrize("B,H,Hk,N,D,rot", [(2, 33, 8, 45, 112, 112), (1, 40, 1, 130, 64, 64), (3, 7, 12, 50, 256, 96),
                                            (1, 65, 0, 17, 66, 34)])
def test_heads_are_divided_where_a_heads_tokens_lie_together(B, H, Hk, N, D, rot, dtype, layout):
    for in_place in (False, True):
        _case(B, H, Hk, N, D, rot, layout, dtype, in_place=in_place)


@pytest.mark.parametrize("layout,dtype,strides,in_place",
                         itertools.product(["half", "interleaved"], ["bf16", "f32"], ["plain", "token", "odd"], [False, True]))
@pytest.mark.parametrize("D,rot", [(112, 56), (64, 20), (128, 70), (128, 94), (64, 62), (66, 36), (40, 24), (24, 24)])
def test_parts_that_are_no_multiple_of_an_access(D, rot, layout, dtype, strides, in_place):
    _case(2, 5, 3, 41, D, rot, layout, dtype, strides=strides, in_place=in_place, backward=rot == 56)


def test_more_heads_than_groups_may_be():
    _case(1, 66000, 1, 2, 64, 64, "half", "bf16")


def test_misaligned_pointer_takes_the_general_path():
    _case(1, 3, 2, 11, 128, 128, "half", "bf16", offset=1)
    _case(1, 3, 2, 11, 128, 64, "interleaved", "f32", offset=1)


def test_gradient_against_differences():
    """<g, R(x + h e) - R(x - h e)> / 2h = (R^T g)_e: the map is linear, so differences are exact
    but for float32 roundings of two sums of 2 * 3 * 5 * 16 products."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((2, 3, 5, 16), generator=g, device="cuda")
    w = torch.randn((2, 3, 5, 16), generator=g, device="cuda")
    pos = torch.arange(10, device="cuda", dtype=torch.int32).reshape(2, 5) * 37
    for layout in ("half", "interleaved"):
        plan = sva.rotary_plan(16, 8, layout, scaling="yarn", factor=4.0, original_len=64)
        grad, _ = sva.rotary(plan, pos, w, backward=True)
        for at in ((0, 0, 0, 0), (1, 2, 4, 7), (0, 1, 3, 5), (1, 0, 2, 12)):
            up, down = x.clone(), x.clone()
            up[at] += 0.5
            down[at] -= 0.5
            d = (sva.rotary(plan, pos, up)[0].double() - sva.rotary(plan, pos, down)[0].double())
            want = float((d * w.double()).sum())
            # results of size up to |x| m (about 6) round at 2^-24 of that, twice per nonzero difference
            assert abs(float(grad[at]) - want) <= 4 * 6 * 2.0 ** -22 * float(w.abs().max())


def test_inf_and_nan_stay_in_their_pair():
    plan = sva.rotary_plan(64, 32, "half")
    x = torch.ones((1, 1, 4, 64), device="cuda", dtype=torch.bfloat16)
    x[0, 0, 1, 3] = float("inf")
    x[0, 0, 2, 40] = float("nan")
    y, _ = sva.rotary(plan, torch.arange(4, device="cuda", dtype=torch.int32)[None], x)
    bad = (~torch.isfinite(y)).nonzero().tolist()
    assert bad == [[0, 0, 1, 3], [0, 0, 1, 19], [0, 0, 2, 40]]
