"""sva_layer_norm on float32 rows whose first channel is far from the others: these keep
their digits."""
import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import layer_norm as oln

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24                       # half a step of float32, relative


@pytest.mark.parametrize("C", [96, 320, 512, 777, 1001, 2240, 4096, 6141, 6144, 8192, 16384])
@pytest.mark.parametrize("far", [1e3, -1e4, 1e5])
def test_a_first_channel_far_from_the_others(C, far):
    say(f"[layer norm] C={C} first channel {far}")
    g = np.random.default_rng(C)
    x, w, b = (g.standard_normal(s).astype(np.float32) for s in ((2, 5, C), (C,), (C,)))
    x[..., 0] = far
    x[1, 1:] += np.float32(300.0)                        # a mean that is far from zero too
    y, mean, rstd = (t.double().cpu().numpy() for t in sva.layer_norm(*(torch.from_numpy(t).cuda() for t in (x, w, b)),
                                                                      want_stats=True))
    x64, w64, b64 = (t.astype(np.float64) for t in (x, w, b))
    want, m, r = oln.forward(x64, w64, b64, 1e-5)
    m, r = m[..., None], r[..., None]
    dev = np.abs(x64 - m)
    # A deviation is rounded twice, from a mean that is off by half a step of itself and, where it is corrected by
    # the sum of the deviations, by that sum's error: chains of up to 40 additions and two products, each U of
    # a deviation in the mean.  Nothing of it grows with a deviation that is not this channel's own.
    d_err = 2 * U * dev + 42 * U * dev.mean(-1, keepdims=True) + 2 * U * np.abs(m)
    # squares: of deviations that are off by that (44 U of the root at most, its mean part being what it is of a
    # root mean square), 102 additions, half of those in the root, and four roundings
    r_err = (44 + 51 + 4) * U + 2 * U * np.abs(m) * r
    assert (np.abs(mean[..., None] - m) <= 42 * U * dev.mean(-1, keepdims=True) + 2 * U * np.abs(m)).all()
    assert (np.abs(rstd[..., None] - r) <= r_err * r).all()
    tol = np.abs(w64) * r * (d_err + dev * (r_err + U)) + U * np.abs(want)
    off = np.abs(y - want)
    assert (off <= 1.001 * tol).all(), (off / tol).max()
