"""The workspace of layer norm's gradients with shared weights: many short entries whose rows follow
each other need the sums of one entry's workgroups, not a row of sums for each entry."""
import pytest

import paper_2606_23743_amd as sva
from paper_2606_23743_amd import _layer, _lib

from .test_side_allocation import Tensor, World

pytestmark = pytest.mark.cpu

torch = pytest.importorskip("torch")


def test_entries_of_one_row_are_one_entry():
    for batch, channels in ((4_000_000, 1024), (70_000, 4096), (2000, 64)):
        assert sva.layer_norm_backward_workspace(batch, 1, channels) == sva.layer_norm_backward_workspace(1, batch, channels)
    # rows of an entry that are apart still need sums of their own, and so do entries' own weights
    assert sva.layer_norm_backward_workspace(70_000, 2, 4096) == 70_000 * 2 * 4096 * 4
    assert sva.layer_norm_backward_workspace(4, 500, 4096, per_entry=True) > 0


class Rows(Tensor):
    """A tensor [B, N, C] of given strides."""

    def __init__(self, shape, strides):
        super().__init__(shape, torch.bfloat16)
        self.strides = strides

    def stride(self, d=None):
        return self.strides if d is None else self.strides[d]


@pytest.mark.parametrize("apart", [False, True])
def test_the_call_allocates_what_its_strides_need(monkeypatch, apart):
    w = World()
    monkeypatch.setattr(_lib, "_torch_module", w.torch)
    monkeypatch.setattr(_layer, "_norm_bytes", {})
    monkeypatch.setattr(_lib, "load", lambda *a: w.lib)          # (workspaces: the library's own)
    B, N, C = 3000, 7, 64
    x = Rows((B, N, C), ((2 if apart else 1) * N * C, C, 1))
    stat = w.t(B, N, dtype=torch.float32)
    w.made.clear()
    _layer.layer_norm_backward(x, x, stat, stat, dx=x)
    scratch = [t for t in w.made if t.dtype == torch.uint8]
    want = sva.layer_norm_backward_workspace(B, N, C) if apart else sva.layer_norm_backward_workspace(1, B * N, C)
    assert [t.numel() for t in scratch] == [want] and (want > 1 << 20) == apart

