"""Refusals of the layer norm, rotary-axes and cross-attention entry points, before any
HIP call: the C ABI with addresses that are never dereferenced, and the binding with host
tensors; workspaces; which stream the memory of these calls belongs to."""
import ctypes
import inspect
import math

import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import rotary_axes as oaxes
from paper_2606_23743_amd import _layer, _lib
from paper_2606_23743_amd._lib import Cross, Heads, LayerNormParams, Positions, RotaryParams, RotarySpec, Rows

from .test_side_allocation import World

pytestmark = pytest.mark.cpu

torch = pytest.importorskip("torch")

A, MB = 1 << 30, 1 << 24
OK, BAD, SHAPE, ALIGN, UNSUP = (_lib.SVA_OK, _lib.SVA_ERR_INVALID_ARG, _lib.SVA_ERR_SHAPE, _lib.SVA_ERR_ALIGNMENT,
                                _lib.SVA_ERR_UNSUPPORTED)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def heads(at, h, n, d):
    return Heads(at, h, h * n * d, n * d, d)


def test_new_symbols_are_declared():
    assert set(_lib.header_functions()) >= {
        "sva_rotary_axes_frequencies", "sva_rotary_axes", "sva_layer_norm", "sva_layer_norm_backward_workspace",
        "sva_layer_norm_backward", "sva_cross_attention_workspace", "sva_cross_attention",
        "sva_cross_attention_backward_workspace", "sva_cross_attention_backward"}


# ------------------------------------------------------------------ rotary axes

@pytest.mark.parametrize("kw", [dict(sections=(20, 18, 18)), dict(sections=(16, 24, 24), base=500000.0),
                                dict(sections=(3, 5), base=(10000.0, 100.0)), dict(sections=(7,), scaling="ntk", factor=4.0),
                                dict(sections=(8, 8, 8, 8), scaling="linear", factor=(1.0, 2.0, 2.0, 1.0)),
                                dict(sections=(16, 16), scaling="yarn", factor=4.0, original_len=(64, 1024))])
def test_axes_frequencies_match_the_oracle(kw):
    f, axis, m = oaxes.ladders(**kw)
    plan = sva.rotary_axes_plan(128, layout="interleaved", device="cpu", **kw)
    # both are float64: a few roundings of pow and exp
    assert np.abs(plan["freq"].numpy() / f - 1).max() < 1e-13
    assert plan["axis"].tolist() == axis.tolist() and math.isclose(plan["magnitude"], m, rel_tol=1e-15)
    assert plan["axes"] == len(kw["sections"]) and plan["rot_dim"] == 2 * sum(kw["sections"])


def test_axes_frequencies_refusals(lib):
    freq, axis, mag = (ctypes.c_double * 512)(), (ctypes.c_int32 * 512)(), ctypes.c_double()

    def call(rots, count=None, **kw):
        specs = (RotarySpec * len(rots))(*(RotarySpec(**{**dict(rot_dim=r, scaling=0, base=1e4, factor=1.0, original_len=0.0,
                                                                beta_fast=32.0, beta_slow=1.0, magnitude=0.0), **kw})
                                           for r in rots))
        return lib.sva_rotary_axes_frequencies(specs, len(rots) if count is None else count, freq, axis, ctypes.byref(mag))

    assert call([2, 510]) == OK and call([512]) == OK
    assert call([0, 4]) == BAD and call([3]) == BAD and call([4], count=0) == BAD and call([8], base=1.0) == BAD
    assert call([256, 258]) == UNSUP and call([2] * 9) == UNSUP
    specs = (RotarySpec * 2)(*(RotarySpec(8, 3, 1e4, f, 64.0, 32.0, 1.0, 0.0) for f in (2.0, 4.0)))
    assert lib.sva_rotary_axes_frequencies(specs, 2, freq, axis, ctypes.byref(mag)) == BAD       # two magnitudes
    assert lib.sva_rotary_axes_frequencies(None, 1, freq, axis, ctypes.byref(mag)) == BAD


def test_rotary_axes_refusals(lib):
    B, H, N, D = 2, 4, 8, 64
    good = dict(batch=B, tokens=N, head_dim=D, rot_dim=D, layout=0, dtype=0, backward=0, magnitude=1.0)
    gpos = dict(data=A, type=0, axes=3, stride_b=3 * N, stride_n=3, stride_a=1)

    def call(freq=A, axis=A, pos=None, qi=None, qo=None, k=True, **kw):
        ki, ko = (heads(A + 2 * MB, 2, N, D), heads(A + 3 * MB, 2, N, D)) if k else (None, None)
        return lib.sva_rotary_axes(RotaryParams(**{**good, **kw}), freq, axis, Positions(**{**gpos, **(pos or {})}),
                                   qi or heads(A, H, N, D), qo or heads(A + MB, H, N, D), ki, ko, None)

    for kw in (dict(freq=None), dict(axis=None), dict(pos=dict(data=None)), dict(pos=dict(type=2)), dict(pos=dict(axes=0)),
               dict(pos=dict(stride_b=-1)), dict(pos=dict(stride_n=-1)), dict(pos=dict(stride_a=-1)), dict(batch=0),
               dict(rot_dim=66), dict(layout=2), dict(dtype=3), dict(magnitude=math.inf), dict(qo=heads(A + 64, H, N, D))):
        assert call(**kw) == BAD, kw
    assert call(pos=dict(axes=9)) == UNSUP and call(head_dim=1026) == UNSUP
    assert call(pos=dict(stride_n=1 << 31)) == SHAPE and call(pos=dict(stride_a=1 << 32)) == SHAPE
    assert call(pos=dict(stride_b=1 << 41)) == SHAPE and call(batch=1 << 20, tokens=1 << 20) == SHAPE
    assert call(freq=A + 4) == ALIGN and call(axis=A + 2) == ALIGN and call(pos=dict(data=A + 2)) == ALIGN
    assert lib.sva_rotary_axes(RotaryParams(**good), A, A, None, heads(A, H, N, D), heads(A + MB, H, N, D), None, None,
                               None) == BAD


# ------------------------------------------------------------------- layer norm

NORM = dict(batch=2, tokens=5, channels=64, dtype=0, weight_dtype=1, per_entry=0, unit_offset=0, weight_stride_b=0,
            bias_stride_b=0, eps=1e-5)


def rows(at, n=5, c=64):
    return Rows(at, n * c, c)


def test_layer_norm_refusals(lib):
    def fwd(x=rows(A), w=A, b=A, y=rows(A + MB), mean=A, rstd=A, **kw):
        return lib.sva_layer_norm(LayerNormParams(**{**NORM, **kw}), x, w, b, y, mean, rstd, None)

    def bwd(dy=rows(A), x=rows(A + MB), w=A, mean=A, rstd=A, ws=A, wb=1 << 30, dx=rows(A + 2 * MB), dw=A, db=A + MB, **kw):
        return lib.sva_layer_norm_backward(LayerNormParams(**{**NORM, **kw}), dy, x, w, mean, rstd, ws, wb, dx, dw, db, None)

    for f in (fwd, bwd):
        for kw in (dict(batch=0), dict(tokens=0), dict(channels=0), dict(dtype=2), dict(weight_dtype=-1), dict(eps=0.0),
                   dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e-40), dict(weight_stride_b=-1), dict(x=None),
                   dict(x=Rows(None, 0, 0)), dict(x=Rows(A, -1, 64))):
            assert f(**kw) == BAD, kw
        assert f(channels=16385) == UNSUP
        assert f(batch=1 << 16, tokens=1 << 15) == SHAPE and f(x=Rows(A, 1 << 62, 1 << 60)) == SHAPE
        assert f(batch=1 << 23, tokens=2, per_entry=1, x=Rows(A, 0, 0), **({"y": Rows(A + MB, 128, 64)} if f is fwd else
                 {"dy": Rows(A, 0, 0), "dx": Rows(A + (1 << 40), 128, 64)})) == SHAPE          # more entries than a launch takes
        assert f(w=A + 2) == ALIGN and f(x=rows(A + 1)) == ALIGN and f(mean=A + 2) == ALIGN and f(rstd=A + 1) == ALIGN
    assert fwd(b=A + 1) == ALIGN
    assert fwd(y=Rows(A + MB, 0, 64)) == BAD                       # an output that repeats itself
    assert fwd(y=Rows(A + MB, 5 * 64, 32)) == BAD                  # its rows overlap
    assert fwd(y=rows(A + 64)) == BAD                              # overlaps x without being it
    for kw in (dict(mean=None), dict(rstd=None), dict(dx=rows(A + 64)), dict(dx=rows(A + MB + 64)), dict(dw=A, db=A)):
        assert bwd(**kw) == BAD, kw
    assert bwd(dw=A + 2) == ALIGN
    many = dict(tokens=900, dy=rows(A, 900), x=rows(A + MB, 900), dx=rows(A + 2 * MB, 900))   # workgroups to be joined
    assert bwd(**many, ws=None) == BAD and bwd(**many, wb=16) == SHAPE and bwd(**many, ws=A + 128) == ALIGN
    assert lib.sva_layer_norm(None, rows(A), None, None, rows(A + MB), None, None, None) == BAD


def test_layer_norm_workspace(lib):
    need = ctypes.c_size_t()
    for kw in (dict(), dict(batch=1, tokens=63240, channels=4096), dict(batch=64, tokens=1, per_entry=1),
               dict(batch=3, tokens=7801, channels=1001), dict(batch=1, tokens=1, channels=16384)):
        assert lib.sva_layer_norm_backward_workspace(LayerNormParams(**{**NORM, **kw}), need) == OK
        p = {**NORM, **kw}
        # a row of sums for weight and bias for each workgroup: never more than there are rows
        assert need.value <= p["batch"] * p["tokens"] * p["channels"] * 8
        assert need.value <= (4096 + p["batch"]) * p["channels"] * 8
    assert lib.sva_layer_norm_backward_workspace(LayerNormParams(**NORM), None) == BAD
    assert sva.layer_norm_backward_workspace(64, 1, 128, per_entry=True) == 0      # an entry's only row
    # as many entries as a launch takes, one more, and as many rows that are one entry's
    most = {**NORM, "batch": 1 << 22, "tokens": 1, "channels": 8}
    assert lib.sva_layer_norm_backward_workspace(LayerNormParams(**{**most, "per_entry": 1}), need) == OK
    assert lib.sva_layer_norm_backward_workspace(LayerNormParams(**{**most, "batch": (1 << 22) + 1, "per_entry": 1}), need) == SHAPE
    assert lib.sva_layer_norm_backward_workspace(LayerNormParams(**{**most, "batch": (1 << 22) + 1, "per_entry": 0}), need) == OK


# -------------------------------------------------------------- cross attention

CROSS = dict(batch=2, heads=4, kv_heads=2, queries=5, keys=9, head_dim=64, softmax_scale=0.0)


def test_cross_attention_refusals(lib):
    N, M, D = 5, 9, 64
    q, k, v, o = heads(A, 4, N, D), heads(A + MB, 2, M, D), heads(A + 2 * MB, 2, M, D), heads(A + 3 * MB, 4, N, D)
    g, dq, dk, dv = heads(A + 4 * MB, 4, N, D), heads(A + 5 * MB, 4, N, D), heads(A + 6 * MB, 2, M, D), heads(A + 7 * MB, 2, M, D)

    def fwd(q=q, k=k, v=v, lens=A, mask=A, mb=M, ws=A, wb=1 << 40, out=o, lse=A, **kw):
        return lib.sva_cross_attention(Cross(**{**CROSS, **kw}), q, k, v, lens, mask, mb, ws, wb, out, lse, None)

    def bwd(dout=g, q=q, k=k, v=v, out=o, lse=A, lens=A, mask=A, mb=M, ws=A, wb=1 << 40, dq=dq, dk=dk, dv=dv, **kw):
        return lib.sva_cross_attention_backward(Cross(**{**CROSS, **kw}), dout, q, k, v, out, lse, lens, mask, mb, ws, wb, dq,
                                                dk, dv, None)

    for f in (fwd, bwd):
        for kw in (dict(batch=0), dict(heads=0), dict(kv_heads=0), dict(queries=0), dict(keys=0), dict(softmax_scale=math.nan),
                   dict(softmax_scale=math.inf), dict(softmax_scale=1e-40), dict(softmax_scale=3e38), dict(mb=-1),
                   dict(q=None), dict(k=Heads(None, 2, 0, 0, 0)), dict(v=Heads(A, 2, -64, 64, 64)), dict(ws=None)):
            assert f(**kw) == BAD, kw
        for kw in (dict(heads=3), dict(k=heads(A + MB, 4, M, D)), dict(q=heads(A, 2, N, D)), dict(queries=1 << 29),
                   dict(keys=1 << 30), dict(wb=16), dict(mb=1 << 41), dict(k=Heads(A, 2, 1 << 62, M * D, D))):
            assert f(**kw) == SHAPE, kw
        for kw in (dict(q=heads(A + 8, 4, N, D)), dict(v=Heads(A, 2, 2 * M * D, M * D + 4, D)), dict(lens=A + 2),
                   dict(lse=A + 2), dict(ws=A + 128)):
            assert f(**kw) == ALIGN, kw
        assert f(head_dim=80) == UNSUP and f(head_dim=256) == UNSUP
        assert f(batch=1 << 23, heads=1, kv_heads=1, queries=1, keys=1) == SHAPE    # more masks than a launch takes
        assert f(batch=1 << 25, heads=1, kv_heads=1, queries=1, keys=1, mask=None) == SHAPE
    for t in (q, k, v):
        assert fwd(out=Heads(t.data, 4, 4 * N * D, N * D, D)) == BAD
    assert fwd(out=Heads(A + 3 * MB, 4, 4 * N * D, 0, D)) == BAD            # an output that repeats itself
    assert bwd(lse=None) == BAD and bwd(dout=None) == BAD
    assert bwd(dk=dv) == BAD and bwd(dq=Heads(g.data, 4, 4 * N * D, N * D, D)) == BAD
    assert bwd(dv=Heads(A + 7 * MB, 2, 0, M * D, D)) == BAD
    assert lib.sva_cross_attention(None, q, k, v, None, None, 0, None, 0, o, None, None) == BAD


def test_cross_attention_workspace(lib):
    need = ctypes.c_size_t()
    p = Cross(**CROSS)
    assert lib.sva_cross_attention_workspace(p, 0, need) == OK and need.value == 0       # nothing is divided
    assert lib.sva_cross_attention_workspace(p, 1, need) == OK and 2 * 4 + 2 * 4 <= need.value <= 1024
    assert lib.sva_cross_attention_backward_workspace(p, 0, need) == OK and need.value >= 2 * 4 * 5 * 8
    assert lib.sva_cross_attention_workspace(p, 0, None) == BAD
    for d in (64, 112, 128):
        for n in (1, 17, 5000):
            for m in (1, 300, 111600):
                for h in (1, 8, 40):
                    # rows of a part are at most the 1,024 workgroups' 128; keys likewise, dK and dV
                    kw = dict(batch=1, heads=h, kv_heads=h, queries=n, keys=m, head_dim=d)
                    a = sva.cross_attention_workspace(**kw)
                    b = sva.cross_attention_workspace(**kw, backward=True)
                    assert a <= 1024 * 128 * (d + 3) * 4 + 4096
                    assert b <= 1024 * 128 * 3 * d * 4 + h * n * 8 + 2 * h * m * d * 4 + 4096
    with pytest.raises(sva.SvaError):
        sva.cross_attention_workspace(1, 3, 2, 1, 1, 64)


# ------------------------------------------------------------------- the binding

def test_binding_refuses_host_tensors_and_wrong_arguments():
    bf = torch.bfloat16
    x = torch.zeros((2, 3, 64), dtype=bf)
    q, k = torch.zeros((2, 4, 3, 64), dtype=bf), torch.zeros((2, 2, 5, 64), dtype=bf)
    st = torch.zeros((2, 3))
    plan = sva.rotary_axes_plan(64, (8, 8), device="cpu")
    for f in (lambda: sva.layer_norm(x), lambda: sva.layer_norm_backward(x, x, st, st), lambda: sva.cross_attention(q, k, k),
              lambda: sva.cross_attention_backward(q, q, k, k, q, st),
              lambda: sva.rotary_axes(plan, torch.zeros((2, 3, 2), dtype=torch.int32), q)):
        with pytest.raises(ValueError, match="device tensor"):
            f()
    with pytest.raises(TypeError):
        sva.layer_norm(x.to(torch.float16))
    with pytest.raises(ValueError):
        sva.layer_norm(x[0])
    with pytest.raises(ValueError):
        sva.layer_norm_backward(x, x[0], st, st)
    with pytest.raises(ValueError, match="layout"):
        sva.rotary_axes_plan(64, (8,), layout="third", device="cpu")
    with pytest.raises(ValueError, match="scaling"):
        sva.rotary_axes_plan(64, (8,), scaling="cubic", device="cpu")
    with pytest.raises(ValueError, match="more than head_dim"):
        sva.rotary_axes_plan(64, (16, 17), device="cpu")
    with pytest.raises(ValueError, match="pairs"):
        sva.rotary_axes_plan(64, (16, 0), device="cpu")
    with pytest.raises(ValueError, match="one value or 2"):
        sva.rotary_axes_plan(64, (8, 8), base=(1e4, 1e4, 1e4), device="cpu")


@pytest.fixture
def world(monkeypatch):
    w = World()
    monkeypatch.setattr(_lib, "_torch_module", w.torch)
    monkeypatch.setattr(_lib, "load", lambda *a: w.lib)
    monkeypatch.setattr(_layer, "_cross_bytes", {})
    return w


def calls(w):
    """name -> (call that leaves everything to be allocated, outputs, whether it has a workspace)."""
    i32, f32, f64 = torch.int32, torch.float32, torch.float64
    x, st = w.t(2, 900, 64), w.t(2, 900, dtype=f32)
    q, k = w.t(1, 4, 3, 64), w.t(1, 2, 5000, 64)
    plan = {"head_dim": 64, "rot_dim": 64, "layout": "half", "magnitude": 1.0, "axes": 2, "freq": w.t(32, dtype=f64),
            "axis": w.t(32, dtype=i32)}
    return {
        "rotary_axes": (lambda **kw: _layer.rotary_axes(plan, w.t(1, 3, 2, dtype=f32), q, w.t(1, 2, 3, 64), **kw), 2, False),
        "layer_norm": (lambda **kw: _layer.layer_norm(x, w.t(64, dtype=f32), want_stats=True, **kw), 3, False),
        "layer_norm_backward": (lambda **kw: _layer.layer_norm_backward(x, x, st, st, **kw), 3, True),
        "cross_attention": (lambda **kw: _layer.cross_attention(q, k, k, w.t(1, dtype=i32), want_lse=True, **kw), 2, True),
        "cross_attention_backward":
            (lambda **kw: _layer.cross_attention_backward(q, q, k, k, q, w.t(1, 4, 3, dtype=f32), **kw), 3, True),
    }


CALLS = ["rotary_axes", "layer_norm", "layer_norm_backward", "cross_attention", "cross_attention_backward"]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("handle", [False, True])
def test_memory_belongs_to_the_stream_that_uses_it_first(world, name, handle):
    call, outputs, workspace = calls(world)[name]
    world.made.clear()
    got = call(stream=world.side.cuda_stream if handle else world.side)
    assert len(got) == outputs and len(world.made) == outputs + workspace and len(world.current) == 1
    assert all(t.made_on == 200 for t in world.made) and all(100 in t.marks for t in got)
    for kw in ({}, {"stream": world.current[0]}):
        world.made.clear()
        call(**kw)
        assert world.made and all(t.made_on == 100 and not t.marks for t in world.made)


def test_every_call_with_a_stream_is_covered():
    takes = {n for n, f in inspect.getmembers(_layer, inspect.isfunction)
             if f.__module__ == _layer.__name__ and not n.startswith("_") and "stream" in inspect.signature(f).parameters}
    assert takes == set(CALLS)
