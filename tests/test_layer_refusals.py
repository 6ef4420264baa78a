"""Calls of layer norm and cross attention that are refused before any HIP call: values past
float32, launches past 2^32 threads, outputs that share memory with what is read or written
beside them.  Addresses are never dereferenced."""
import pytest

from paper_2606_23743_amd import _lib
from paper_2606_23743_amd._lib import LayerNormParams, Rows

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
