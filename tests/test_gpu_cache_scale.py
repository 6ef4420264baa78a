"""sva_cache_attention at the smallest softmax scales it takes: every logit next to zero, masked keys still out."""
import numpy as np
import pytest

from .gpu_cases import say
from .test_gpu_cache_attention import Case, trees

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("T", [5, 60, 100])
def test_the_smallest_scale_gives_means(fmt, T):
    c = Case(41, 2, 1, 1, T, 64, 64, fmt, [130, 0])
    m = trees(c.g, 2, T)
    m[:, T // 2] = 0                                     # a row that sees cached tokens alone, or nothing
    for scale in (1e-38, 1e-30):
        say(f"[cache attention] scale {scale}")
        out, lse = c.run(mask=m, f32=True, scale=scale)
        out = out.cpu().numpy()
        assert np.isfinite(out).all() and (out[1, 0, T // 2] == 0).all()
        assert torch.isneginf(lse[1, 0, T // 2]) and not torch.isnan(lse).any()
