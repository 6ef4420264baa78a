"""Pins of oracle/rotary.py and oracle/kv_cache.py: closed forms, brute force and
library routines."""
import math

import numpy as np
import pytest

from oracle import kv_cache as okv, rotary as orot

pytestmark = pytest.mark.cpu

torch = pytest.importorskip("torch")


def test_frequencies_by_hand():
    f, m = orot.frequencies(8)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001], rtol=1e-14) and m == 1.0
    f, _ = orot.frequencies(8, scaling="linear", factor=4.0)
    assert np.allclose(f, [0.25, 0.025, 0.0025, 0.00025], rtol=1e-14)
    # NTK keeps the highest frequency and makes the lowest s times longer
    f, _ = orot.frequencies(64, scaling="ntk", factor=8.0)
    g, _ = orot.frequencies(64)
    assert f[0] == 1.0 and math.isclose(f[-1], g[-1] / 8.0, rel_tol=1e-12)
    # by parts: pairs of more than beta_fast turns keep their frequency, those below beta_slow lose s
    f, m = orot.frequencies(128, scaling="yarn", factor=16.0, original_len=4096)
    g, _ = orot.frequencies(128)
    turns = 4096 * g / (2 * math.pi)
    assert np.all(f[turns >= 32] == g[turns >= 32]) and np.allclose(f[turns <= 1], g[turns <= 1] / 16.0)
    assert math.isclose(m, 1 + 0.1 * math.log(16.0))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_by_hand_and_its_transpose(layout):
    x = np.zeros((1, 1, 1, 6))
    x[..., 0] = 1.0                                # first member of pair 0; channels 4, 5 not turned
    x[..., 4:] = (7.0, -3.0)
    f = np.array([math.pi / 2, 0.3])
    y = orot.apply(x, np.array([[1]]), f, 2.0, layout)[0, 0, 0]
    assert np.allclose(y, [0, 0, 2, 0, 7, -3] if layout == "half" else [0, 2, 0, 0, 7, -3], atol=1e-15)
    g = np.random.default_rng(1)
    a, b = g.standard_normal((2, 2, 3, 5, 6))
    pos = g.integers(-50, 50, (2, 5))
    ya = orot.apply(a, pos, f, 1.3, layout)
    tb = orot.apply(b, pos, f, 1.3, layout, backward=True)
    assert math.isclose((ya * b).sum(), (a * tb).sum(), rel_tol=1e-12)


def test_rounding_to_e4m3_is_the_library_cast():
    g = np.random.default_rng(2)
    x = np.concatenate([g.standard_normal(4000) * 10.0 ** g.uniform(-4, 2.4, 4000), okv.e4m3_values()[:127],
                        (okv.e4m3_values()[:126] + okv.e4m3_values()[1:127]) / 2, [0.0, -0.0, 448.0, -448.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(okv.round_e4m3(x), want)


def test_quantised_rows():
    x = np.array([[0.0, 0.0], [448.0, 1.0], [449.0, 1.0], [0.875, -0.4], [1e-30, 0.0]])
    _, s = okv.quantise_rows(x, "e4m3")
    assert s[0] == 1.0 and s[1] == 1.0 and s[2] == 2.0 and s[3] == 2.0 ** -9
    assert 448 * s[4] >= 1e-30 > 224 * s[4]
    c, s = okv.quantise_rows(np.array([[127.0, 0.5, 1.5, -2.5, 100.0], [0, 0, 0, 0, 0.0]]), "int8")
    assert np.array_equal(c, [[127, 0, 2, -2, 100], [0, 0, 0, 0, 0]]) and np.array_equal(s, [1.0, 1.0])


def test_attention_is_the_library_softmax_on_what_is_seen():
    g = np.random.default_rng(3)
    q, k, v = g.standard_normal((4, 8)), g.standard_normal((9, 8)), g.standard_normal((9, 8))
    seen = g.random((4, 9)) < 0.6
    seen[2] = False
    seen[0, 0] = seen[1, 1] = seen[3, 3] = True
    o, lse = okv.attention(q, k, v, seen, 0.3)
    s = torch.from_numpy(0.3 * q @ k.T).masked_fill(torch.from_numpy(~seen), -math.inf)
    keep = [0, 1, 3]
    assert np.allclose(o[keep], (torch.softmax(s, -1) @ torch.from_numpy(v))[keep], rtol=1e-12)
    assert np.allclose(lse[keep], torch.logsumexp(s, -1)[keep], rtol=1e-12)
    assert np.all(o[2] == 0) and lse[2] == -math.inf
