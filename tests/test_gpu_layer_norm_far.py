"""Gradients of sva_layer_norm from rows whose mean times rstd is past float32: what is not
there of a row takes no part."""
import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import layer_norm as oln

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U, UB = 2.0 ** -24, 2.0 ** -8        # half a step of float32 and of bf16, relative


@pytest.mark.parametrize("C", [3, 8, 77, 128, 136, 320, 505, 520, 1001, 1016, 1536, 2049, 4104, 8200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_equal_huge_elements(C, dtype):
    say(f"[layer norm] gradients of constant rows of 1e37, C={C} {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = np.random.default_rng(C)
    x = torch.full((1, 5, C), 1e37, dtype=dt, device="cuda")
    dy = torch.from_numpy(g.standard_normal((1, 5, C)).astype(np.float32)).to(dt).cuda()
    w = torch.from_numpy(g.standard_normal(C).astype(np.float32)).cuda()
    mean, rstd = x[..., 0].float().contiguous(), torch.full((1, 5), 316.0, device="cuda")
    got = [t.double().cpu().numpy() for t in sva.layer_norm_backward(dy, x, mean, rstd, w)]
    dy64, w64 = dy.double().cpu().numpy(), w.double().cpu().numpy()
    want = oln.backward(dy64, x.double().cpu().numpy(), mean.double().cpu().numpy(), rstd.double().cpu().numpy(), w64)
    gabs = np.abs(dy64 * w64)
    # g and its difference from the mean are rounded, the mean is a sum of up to 40 additions; xhat is zero
    tol = 316.0 * U * (4 * gabs + 44 * gabs.mean(-1, keepdims=True)) + 4 * U * np.abs(want[0])
    tol = tol * (1 + UB) + (UB if dtype == "bf16" else U) * np.abs(want[0])
    assert (np.abs(got[0] - want[0]) <= tol).all()
    assert not got[1].any() and (np.abs(got[2] - want[2]) <= 9 * U * np.abs(dy64).sum((0, 1))).all()
