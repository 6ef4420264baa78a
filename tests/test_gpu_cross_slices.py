"""Cross attention on slices of one projection, whose rows interleave, and outputs written into
slices beside them: the same bits as on tensors of their own, and nothing else is written."""
import pytest

import paper_2606_23743_amd as sva

from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("H,kv,N,D", [(4, 4, 150, 64), (8, 2, 70, 128), (5, 1, 1, 112)])
def test_slices_of_one_projection(H, kv, N, D):
    say(f"[cross] slices of one projection, {H}/{kv} heads of {D}, {N} tokens")
    B = 2
    g = torch.Generator(device="cuda").manual_seed(N)
    heads = (H, kv, kv, H, H, H, kv, kv, 1)               # q, k, v, out, dout, dq, dk, dv, and one that is nobody's
    both = torch.randn((B, N, sum(heads), D), generator=g, device="cuda").to(torch.bfloat16)
    cuts = [sum(heads[:i]) for i in range(len(heads) + 1)]
    part = [both[:, :, a:b].transpose(1, 2) for a, b in zip(cuts, cuts[1:])]
    q, k, v, out, dout, dq, dk, dv, rest = part
    own = [t.clone().contiguous() for t in (q, k, v, dout, rest)]
    want, lse = sva.cross_attention(*own[:3], want_lse=True)
    grads = sva.cross_attention_backward(own[3], *own[:3], want, lse)
    sva.cross_attention(q, k, v, out=out, want_lse=True)
    assert torch.equal(out, want)
    sva.cross_attention_backward(dout, q, k, v, out, lse, dq=dq, dk=dk, dv=dv)
    for a, b in zip((dq, dk, dv), grads):
        assert torch.equal(a, b)
    for a, b in zip((q, k, v, dout, rest), own):
        assert torch.equal(a, b)


def test_an_output_over_an_input_is_refused():
    x = torch.zeros((1, 2, 41, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((1, 2, 9, 64), dtype=torch.bfloat16, device="cuda")
    for out in (x[:, :, 1:], x[:, :, :40]):
        with pytest.raises(sva.SvaError):
            sva.cross_attention(x[:, :, :40], k, k, out=out)
