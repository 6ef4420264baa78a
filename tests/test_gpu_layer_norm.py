"""sva_layer_norm and its gradients on the GPU against oracle/layer_norm.py: every way a
row is held, types, strides and alignments, weights shared and per entry, in place."""
import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import layer_norm as oln

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U, UB = 2.0 ** -24, 2.0 ** -8        # half a step of float32 and of bf16, relative


def _tensor(g, shape, dtype, layout="plain", scale=1.0, shift=0.0, offset=0):
    """(device tensor of that layout, its values in float64)."""
    B, N, C = shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.from_numpy((g.standard_normal(shape) * scale + shift).astype(np.float32)).to(dt)
    if layout == "plain":
        y = torch.empty(B * N * C + offset, dtype=dt, device="cuda")[offset:].view(shape)
    elif layout == "wide":                             # a slice of wider rows, entries innermost but one
        y = torch.empty((N, B, C + 24), dtype=dt, device="cuda")[:, :, 8:8 + C].transpose(0, 1)
    else:                                              # odd pitches: no whole 16-byte accesses
        y = torch.empty((B, N, C + 3), dtype=dt, device="cuda")[:, :, 1:1 + C]
    return y.copy_(x), x.double().numpy()


def _weights(g, kind, B, C, wdtype):
    if kind == "none":
        return None, None, None, None
    shape = (B, C) if kind == "entry" else (C,)
    dt = torch.bfloat16 if wdtype == "bf16" else torch.float32
    w, b = (torch.from_numpy(g.standard_normal(shape).astype(np.float32)).to(dt) for _ in range(2))
    dev = [t.cuda() for t in (w, b)]
    if kind == "entry":                                # as slices of one modulation
        both = torch.cat(dev, dim=1)
        dev = [both[:, :C], both[:, C:]]
    return dev[0], dev[1], w.double().numpy(), b.double().numpy()


def _case(B, N, C, dtype="bf16", kind="entry", unit=True, layout="plain", wdtype="f32", scale=1.0, shift=0.0, eps=1e-5,
          in_place=False, offset=0, grads=True):
    g = np.random.default_rng(B * 100 + N + C)
    say(f"[layer norm] B={B} N={N} C={C} {dtype} {kind} {wdtype} {layout}+{offset} unit={unit} scale={scale} shift={shift} "
        f"in_place={in_place}")
    x, x64 = _tensor(g, (B, N, C), dtype, layout, scale, shift, offset)
    w, b, w64, b64 = _weights(g, kind, B, C, wdtype)
    one = 1.0 if unit else 0.0
    before = x.clone()
    y, mean, rstd = sva.layer_norm(x, w, b, eps, unit, y=x if in_place else None, want_stats=True)
    torch.cuda.synchronize()
    want, m64, r64 = oln.forward(x64, w64, b64, eps, one)
    # The mean is off by two steps of itself; by the sum's chain, at most 22 additions of elements (bf16) or of
    # their differences from the first one (float32), or by 42 U of a deviation where waves' means are joined.
    base = np.abs(x64 - (x64[..., :1] if dtype == "f32" else 0.0)).mean(-1)
    mean_tol = 2 * U * np.abs(m64) + 42 * U / r64 + 22 * U * base
    assert (np.abs(mean.double().cpu().numpy() - m64) <= mean_tol).all()
    # squares are summed in chains of at most 96 in a lane, 6 over lanes, 16 over waves, and have two steps of their
    # own: the root is off by half of 120 U and its own three; a mean off by d adds (d rstd)^2 / 2
    r_tol = 63 * U + (mean_tol * r64) ** 2
    assert (np.abs(rstd.double().cpu().numpy() - r64) <= r_tol * r64).all()
    rows = lambda t, none: np.full(C, none) if t is None else t[:, None] if t.ndim == 2 else t  # noqa: E731
    wf = np.abs(rows(w64, 1.0) + (one if w64 is not None else 0.0)) + (2 * U if unit else 0.0)
    xh = np.abs((x64 - m64[..., None]) * r64[..., None])
    tol = (wf * (xh * (r_tol[..., None] + 4 * U) + mean_tol[..., None] * r64[..., None])
           + 2 * U * (np.abs(want) + np.abs(rows(b64, 0.0))))
    out_u = UB if dtype == "bf16" else U
    got = y.double().cpu().numpy()
    assert y.dtype == x.dtype and (np.abs(got - want) <= tol * (1 + out_u) + out_u * np.abs(want) + 1e-38).all(), \
        np.abs(got - want).max()
    if not in_place:
        assert torch.equal(before, x)
    if not grads:
        return
    # the gradient from statistics as float32 holds them
    sm, sr = torch.from_numpy(m64.astype(np.float32)).cuda(), torch.from_numpy(r64.astype(np.float32)).cuda()
    dy, dy64 = _tensor(g, (B, N, C), dtype, layout, offset=offset)
    m32, r32 = m64.astype(np.float32).astype(np.float64), r64.astype(np.float32).astype(np.float64)
    per = kind == "entry"
    dx_want, dw_want, db_want = oln.backward(dy64, x64, m32, r32, w64, one, per)
    keep = dy.clone()
    dx, dw, db = sva.layer_norm_backward(dy, before, sm, sr, w, unit, dx=dy if in_place else None)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(keep, dy) and dx.dtype == x.dtype
    wabs = np.abs(rows(w64, 1.0) + (one if w64 is not None else 0.0))
    gabs, r = np.abs(dy64) * wabs, r32[..., None]
    xa = np.abs((x64 - m32[..., None]) * r)                     # off by 2 U of itself
    m1, m2 = gabs.mean(-1, keepdims=True), (gabs * xa).mean(-1, keepdims=True)
    tol = r * U * (4 * gabs + 44 * m1 + xa * 52 * m2) + 4 * U * np.abs(dx_want)
    got = dx.double().cpu().numpy()
    assert (np.abs(got - dx_want) <= tol * (1 + out_u) + out_u * np.abs(dx_want) + 1e-38).all(), np.abs(got - dx_want).max()
    # whatever the order, a sum of n terms is off by at most n U of their magnitudes' sum
    over, n = ((1,), N) if per else ((0, 1), B * N)
    for a, t, size in ((dw, dw_want, np.abs(dy64) * xa), (db, db_want, np.abs(dy64))):
        assert a.dtype == torch.float32 and a.shape == t.shape
        assert (np.abs(a.double().cpu().numpy() - t) <= (n + 4) * U * size.sum(axis=over) + 1e-38).all()


# 16 lanes to a row, 32, 64, a workgroup with one piece a lane and two, up to sixteen waves
@pytest.mark.parametrize("C", [1, 2, 7, 8, 64, 127, 128, 136, 250, 256, 264, 505, 512, 513, 520, 1001, 1024, 2040, 2048, 2049,
                               2056, 4096, 4104, 6144, 8192, 8200, 16383, 16384])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_channels(C, dtype):
    _case(2, 5, C, dtype)


@pytest.mark.parametrize("kind,unit,wdtype", [("none", False, "f32"), ("shared", False, "f32"), ("shared", True, "bf16"),
                                              ("entry", False, "bf16"), ("entry", True, "f32")])
@pytest.mark.parametrize("C", [40, 77, 384, 1400])
@pytest.mark.parametrize("layout", ["plain", "wide", "odd"])
def test_weights_and_strides(kind, unit, wdtype, C, layout):
    _case(3, 9, C, "bf16" if C % 8 else "f32", kind, unit, layout, wdtype)


@pytest.mark.parametrize("C", [64, 200, 333, 1024, 2240])
@pytest.mark.parametrize("dtype,layout", [("bf16", "plain"), ("f32", "odd"), ("bf16", "wide")])
def test_in_place(C, dtype, layout):
    _case(2, 6, C, dtype, "shared", False, layout, in_place=True)


@pytest.mark.parametrize("B,N", [(1, 1), (1, 17), (65, 1), (3, 3000), (1, 9001), (200, 33)])
@pytest.mark.parametrize("C,kind", [(96, "shared"), (96, "entry"), (640, "shared"), (640, "entry")])
def test_rows(B, N, C, kind):
    _case(B, N, C, "bf16", kind)


@pytest.mark.parametrize("C", [48, 320, 1536])
def test_means_far_from_zero_and_small_deviations(C):
    _case(2, 4, C, "f32", scale=1.0, shift=1000.0)
    _case(2, 4, C, "f32", scale=1e-3, shift=0.0, eps=1e-6)
    _case(2, 4, C, "bf16", scale=1e4)
    _case(2, 4, C, "f32", scale=0.0, shift=3.0)          # constant rows: the bias alone


def test_misaligned_pointers():
    for dtype in ("bf16", "f32"):
        for C in (64, 1024, 1001):
            _case(2, 5, C, dtype, offset=1)


def test_only_one_of_the_sums_and_none():
    x = torch.randn((2, 700, 128), device="cuda")
    dy = torch.randn_like(x)
    _, mean, rstd = sva.layer_norm(x, want_stats=True)
    dx, dw, db = sva.layer_norm_backward(dy, x, mean, rstd)
    only = torch.full((128,), -7.0, device="cuda")
    dx2, dw2, db2 = sva.layer_norm_backward(dy, x, mean, rstd, want_weight=False, dweight=only)
    assert torch.equal(dx, dx2) and torch.equal(dw2, dw) and db2 is None
    dx3, a, b = sva.layer_norm_backward(dy, x, mean, rstd, want_weight=False)
    assert torch.equal(dx, dx3) and a is None and b is None
    _, pw, pb = sva.layer_norm_backward(dy, x, mean, rstd, per_entry=True)
    assert pw.shape == (2, 128) and torch.allclose(pw.sum(0), dw, rtol=0, atol=1e-3) and torch.allclose(pb.sum(0), db, rtol=0, atol=1e-3)


def test_inputs_that_repeat_themselves_and_far_rows():
    """x of one row for all tokens (stride 0); rows past 2^31 elements."""
    g = np.random.default_rng(9)
    row = torch.from_numpy(g.standard_normal((1, 1, 96)).astype(np.float32)).cuda()
    x = row.expand(3, 50, 96)
    y, _, _ = sva.layer_norm(x, y=torch.empty((3, 50, 96), device="cuda"))
    alone, _, _ = sva.layer_norm(row)
    assert torch.equal(y, alone.expand(3, 50, 96))
    big = torch.empty((1 << 31) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((2, 2, 512), (1 << 30, 1 << 30, 1))
    data = torch.randn((2, 2, 512), device="cuda").to(torch.bfloat16)
    data[0, 1] = data[1, 0]                              # one place
    far.copy_(data)
    out = torch.empty((2, 2, 512), dtype=torch.bfloat16, device="cuda")
    assert torch.equal(sva.layer_norm(far, y=out)[0], sva.layer_norm(data)[0])


def test_a_bad_row_stays_alone():
    x = torch.randn((1, 9, 320), device="cuda")
    x[0, 3, 5], x[0, 6, 7] = float("inf"), float("nan")
    y, mean, rstd = sva.layer_norm(x, want_stats=True)
    good = [0, 1, 2, 4, 5, 7, 8]
    assert torch.isfinite(y[0, good]).all() and torch.isnan(y[0, 6]).all() and not torch.isfinite(y[0, 3]).any()
    dx, _, _ = sva.layer_norm_backward(torch.ones_like(x), x, mean, rstd)
    assert torch.isfinite(dx[0, good]).all()


def test_gradient_against_differences():
    """Central differences of the 64-bit forward; h^2 times a third derivative, below 1e-7 here."""
    g = np.random.default_rng(4)
    x, dy, w = g.standard_normal((1, 2, 24)), g.standard_normal((1, 2, 24)), g.standard_normal(24)
    x, dy, w = (t.astype(np.float32).astype(np.float64) for t in (x, dy, w))
    t = lambda v: torch.from_numpy(v.astype(np.float32)).cuda()  # noqa: E731
    _, mean, rstd = sva.layer_norm(t(x), t(w), None, 1e-3, want_stats=True)
    dx, dw, _ = sva.layer_norm_backward(t(dy), t(x), mean, rstd, t(w))
    h = 1e-4

    def slope(v, at):
        keep = v[at]
        v[at] = keep + h
        up = (oln.forward(x, w, None, 1e-3)[0] * dy).sum()
        v[at] = keep - h
        down = (oln.forward(x, w, None, 1e-3)[0] * dy).sum()
        v[at] = keep
        return (up - down) / (2 * h)

    # values of up to 10 in float32, by some fifty roundings
    for at in np.ndindex(1, 2, 24):
        assert abs(float(dx[at]) - slope(x, at)) < 50 * U * 10 + 1e-6
    for at in np.ndindex(24):
        assert abs(float(dw[at]) - slope(w, at)) < 50 * U * 10 + 1e-6


def test_same_bits_twice_and_on_a_side_stream():
    x = torch.randn((2, 5000, 520), device="cuda").to(torch.bfloat16)
    dy = torch.randn((2, 5000, 520), device="cuda").to(torch.bfloat16)
    w = torch.randn(520, device="cuda")

    def step(s):
        y, m, r = sva.layer_norm(x, w, w, want_stats=True, stream=s)
        return [y, m, r, *sva.layer_norm_backward(dy, x, m, r, w, stream=s)]

    want = step(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(want, got, step(None)):
        assert torch.equal(a, b) and torch.equal(a, c)
