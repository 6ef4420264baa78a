"""Calls of layer norm and cross attention that are refused before any HIP call: values past
float32, launches past 2^32 threads, outputs that share memory with what is read or written
beside them.  Addresses are never dereferenced."""
import pytest

from paper_2606_23743_amd import _lib
from paper_2606_23743_amd._lib import Cross, Heads, LayerNormParams, Rows

pytestmark = pytest.mark.cpu

A, MB = 1 << 30, 1 << 24
OK, BAD, SHAPE = _lib.SVA_OK, _lib.SVA_ERR_INVALID_ARG, _lib.SVA_ERR_SHAPE
NORM = dict(batch=2, tokens=5, channels=64, dtype=0, weight_dtype=1, per_entry=0, unit_offset=0, weight_stride_b=0,
            bias_stride_b=0, eps=1e-5)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def rows(at, n=5, c=64):
    return Rows(at, n * c, c)


@pytest.mark.parametrize("eps", [3.5e38, 1e300])
def test_an_eps_past_float32(lib, eps):
    """As float32 it would be infinite, and every row its bias."""
    p = LayerNormParams(**{**NORM, "eps": eps})
    assert lib.sva_layer_norm(p, rows(A), None, None, rows(A + MB + 1), None, None, None) == BAD     # (before y's alignment)
    assert lib.sva_layer_norm_backward_workspace(p, _lib.ctypes.c_size_t()) == BAD


@pytest.mark.parametrize("per_entry", [0, 1])
def test_launches_past_32_bits_of_threads(lib, per_entry):
    """2^22 entries of their own in workgroups of 1,024 threads; one entry fewer, or fewer threads, are a launch."""
    B, need = 1 << 22, _lib.ctypes.c_size_t()

    def asked(batch, channels):
        return lib.sva_layer_norm_backward_workspace(LayerNormParams(**{**NORM, "batch": batch, "tokens": 1, "channels": channels,
                                                                        "per_entry": 1}), need)

    assert asked(B, 16384) == SHAPE and asked(B, 15361) == SHAPE
    assert asked(B - 1, 16384) == OK and asked(B, 15360) == OK and asked(B, 8) == OK
    p = LayerNormParams(**{**NORM, "batch": B, "tokens": 2, "channels": 16384, "per_entry": per_entry})
    x, y = Rows(A, 0, 0), Rows(A + MB, 3 * 16384, 16384)                       # (no pitch of all rows)
    assert lib.sva_layer_norm(p, x, None, None, y, None, None, None) == SHAPE
    assert lib.sva_layer_norm_backward(p, x, x, None, A, A, A, 1 << 60, y, A, A + MB, None) == SHAPE


# ---- cross attention: outputs that share memory ----

B, H, KV, N, M, D = 2, 4, 2, 5, 9, 64


def _cross(**kw):
    """Arguments of both calls, all apart (and the mask and workspace large)."""
    at = iter(A + i * MB for i in range(20))
    q = lambda: _rows(next(at))  # noqa: E731
    k = lambda: Heads(next(at), KV, KV * M * D, M * D, D)  # noqa: E731
    t = dict(q=q(), k=k(), v=k(), out=q(), dout=q(), dq=q(), dk=k(), dv=k(), lse=next(at), lens=next(at), mask=next(at), ws=next(at))
    return {**t, **{n: f(t) for n, f in kw.items()}}


def _rows(at):
    return Heads(at, H, H * N * D, N * D, D)


def _moved(x, elements):
    return Heads(x.data + 2 * elements, x.heads, x.stride_b, x.stride_h, x.stride_n)


FORWARD = {
    "out is q one token on": dict(out=lambda t: _moved(t["q"], D)),
    "out is q one token back": dict(out=lambda t: _moved(t["q"], -D)),
    "out is q one head on": dict(out=lambda t: _moved(t["q"], N * D)),
    "out ends in k": dict(out=lambda t: _rows(t["k"].data - 2 * (B * H * N - 1) * D)),
    "out begins at v's last row": dict(out=lambda t: _rows(t["v"].data + 2 * (B * KV * M - 1) * D)),
    "lse in q": dict(lse=lambda t: t["q"].data + 64),
    "lse in out": dict(lse=lambda t: t["out"].data + 64),
    "lse over the lengths": dict(lse=lambda t: t["lens"] - 8),
    "out over the mask": dict(out=lambda t: _rows(t["mask"] + 16 - 2 * B * H * N * D)),
    "workspace in v": dict(ws=lambda t: t["v"].data + 256),
    "workspace over out": dict(ws=lambda t: t["out"].data),
}
BACKWARD = {
    "dq is q one token on": dict(dq=lambda t: _moved(t["q"], D)),
    "dq is dout one token on": dict(dq=lambda t: _moved(t["dout"], D)),
    "dq is out one token back": dict(dq=lambda t: _moved(t["out"], -D)),
    "dk is k one row on": dict(dk=lambda t: _moved(t["k"], D)),
    "dv is v one head on": dict(dv=lambda t: _moved(t["v"], M * D)),
    "dk is dv one row on": dict(dk=lambda t: _moved(t["dv"], D)),
    "dv begins in dq": dict(dv=lambda t: Heads(t["dq"].data + 16, KV, KV * M * D, M * D, D)),
    "dq over the lse": dict(dq=lambda t: _rows(t["lse"])),
    "workspace over dk": dict(ws=lambda t: t["dk"].data),
}


def _forward(lib, t):
    return lib.sva_cross_attention(Cross(B, H, KV, N, M, D, 0.0), t["q"], t["k"], t["v"], t["lens"], t["mask"], M, t["ws"],
                                   1 << 20, t["out"], t["lse"], None)


def _backward(lib, t):
    return lib.sva_cross_attention_backward(Cross(B, H, KV, N, M, D, 0.0), t["dout"], t["q"], t["k"], t["v"], t["out"], t["lse"],
                                            t["lens"], t["mask"], M, t["ws"], 1 << 20, t["dq"], t["dk"], t["dv"], None)


@pytest.mark.parametrize("name", FORWARD)
def test_cross_attention_outputs_apart(lib, name):
    assert _forward(lib, _cross(**FORWARD[name])) == BAD


@pytest.mark.parametrize("name", BACKWARD)
def test_cross_attention_gradients_apart(lib, name):
    assert _backward(lib, _cross(**BACKWARD[name])) == BAD


# ---- layer norm: the same ----

TOKENS = 900                                             # (workgroups to be joined: a workspace)


def _norm(**kw):
    at = iter(A + i * MB for i in range(20))
    t = dict(**{n: rows(next(at), TOKENS) for n in ("x", "y", "dy", "dx")}, **{n: next(at) for n in (
        "w", "b", "mean", "rstd", "dw", "db", "ws")})
    return {**t, **{n: f(t) for n, f in kw.items()}}


NORM_FORWARD = {
    "mean is rstd": dict(mean=lambda t: t["rstd"]),
    "mean ends in rstd": dict(mean=lambda t: t["rstd"] - 4),
    "rstd in y": dict(rstd=lambda t: t["y"].data + 4),
    "mean in x": dict(mean=lambda t: t["x"].data + 4),
    "rstd in the weight": dict(rstd=lambda t: t["w"] + 4),
    "y over the bias": dict(y=lambda t: rows(t["b"], TOKENS)),
    "y ends in the weight": dict(y=lambda t: rows(t["w"] - 2 * 2 * TOKENS * 64 + 2, TOKENS)),
}
NORM_BACKWARD = {
    "the sums are one": dict(dw=lambda t: t["db"]),
    "the sums overlap": dict(dw=lambda t: t["db"] + 4),
    "a sum in dy": dict(dw=lambda t: t["dy"].data),
    "a sum in dx": dict(db=lambda t: t["dx"].data + 4),
    "a sum over the weight": dict(dw=lambda t: t["w"]),
    "dx over the mean": dict(dx=lambda t: rows(t["mean"], TOKENS)),
    "dx over the weight": dict(dx=lambda t: rows(t["w"], TOKENS)),
    "workspace over a sum": dict(ws=lambda t: t["dw"]),
    "workspace over x": dict(ws=lambda t: t["x"].data),
}


@pytest.mark.parametrize("name", NORM_FORWARD)
def test_layer_norm_outputs_apart(lib, name):
    t = _norm(**NORM_FORWARD[name])
    assert lib.sva_layer_norm(LayerNormParams(**{**NORM, "tokens": TOKENS}), t["x"], t["w"], t["b"], t["y"], t["mean"], t["rstd"], None) == BAD


@pytest.mark.parametrize("name", NORM_BACKWARD)
def test_layer_norm_gradients_apart(lib, name):
    t = _norm(**NORM_BACKWARD[name])
    p = LayerNormParams(**{**NORM, "tokens": TOKENS})
    assert lib.sva_layer_norm_backward(p, t["dy"], t["x"], t["w"], t["mean"], t["rstd"], t["ws"], 1 << 20, t["dx"], t["dw"],
                                       t["db"], None) == BAD
