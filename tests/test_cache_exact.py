"""What tests/cache_exact.py can tell apart, on the CPU: mistakes planted in the oracle."""
import numpy as np
import pytest

from . import cache_exact as ce

pytestmark = pytest.mark.cpu

torch = pytest.importorskip("torch")

SIZES = dict(B=2, kv=2, G=2, T=5, D=64, page=64, lengths=[1100, 70])


def _bf16(x):
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()


def by_parts(c, parts):
    """The results with weights times V's scale as a sum of `parts` bf16 values."""
    B, H, T, D = c.B, c.kv * c.G, c.T, c.D
    out = np.zeros((B, H, T, D))
    q, kn, vn = (x.double().numpy() for x in (c.q, c.k_new, c.v_new))
    for b in range(B):
        n, cnt = int(c.lengths[b]), int(c.counts[b])
        at = np.arange(n)
        pages, place = c.table[b][at // c.page], at % c.page
        for h in range(c.kv):
            z = np.ones(n + cnt)
            if c.fmt != "bf16":
                z[:n] = c.cache["v_scale"].double().numpy()[pages, h, place]
            k = np.concatenate((c.rows("k", b, h), kn[b, h, :cnt]))
            v = np.concatenate((c.rows("v", b, h), vn[b, h, :cnt])) / z[:, None]
            seen = np.ones((cnt, n + cnt), bool)
            seen[:, n:] = c.mask[b, :cnt, :cnt] != 0
            for i in range(h * c.G, (h + 1) * c.G):
                s = np.where(seen, c.scale * (q[b, i, :cnt] @ k.T), -np.inf)
                w = np.exp(s - s.max(axis=1, keepdims=True)).astype(np.float32).astype(np.float64)
                wz = (w * z).astype(np.float32).astype(np.float64)
                rest, total = wz.copy(), np.zeros_like(wz)
                for _ in range(parts):
                    part = _bf16(rest)
                    total += part
                    rest -= part
                out[b, i, :cnt] = total @ v / w.sum(axis=1, keepdims=True)
    return out


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_two_parts_are_told_from_three(fmt):
    c = ce.fine_case(3, fmt=fmt, **SIZES)
    want = c.exact()
    two, three = (ce.norm_error(by_parts(c, n), want) for n in (2, 3))
    assert three < ce.FINE_NORM / 4 and two > 1.5 * ce.FINE_NORM


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_whole_cases_are_exact_in_bf16_weights_and_float32_sums(fmt):
    c = ce.whole_case(4, fmt=fmt, **SIZES)
    want = c.exact()
    ce.check_whole(by_parts(c, 1), None, want, True)
    x = c.scale * np.einsum("bhtd,bhsd->bhts", c.q.double().numpy(), np.repeat(c.k_new.double().numpy(), c.G, 1)) / ce.LN2
    assert np.abs(x - np.rint(x)).max() < 1e-12 and np.abs(x).max() <= 1 + 1e-12
    assert np.float32(c.scale * 1.4426950408889634074) == 1.0
    assert float(np.abs(c.values["v"]).max()) == 8.0
    assert set(np.unique(c.values["k"][..., 0])) == {0.0, 1.0}


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("mistake", ["lost unit", "unit twice", "another head's unit", "one key lost", "lost numerator",
                                     "two keys exchanged"])
def test_planted_mistakes_are_seen(mistake, f32):
    c = ce.whole_case(5, fmt="e4m3", **SIZES)
    want = c.exact()
    q = c.q.double().numpy()
    b, h, t = 0, 1, 2
    k, v = c.rows("k", 0, 0), c.rows("v", 0, 0)
    kn, vn = c.k_new.double().numpy()[0, 0], c.v_new.double().numpy()[0, 0]
    on = c.mask[0, t] != 0
    w = np.concatenate((np.exp2(k @ q[b, h, t]), np.exp2(kn @ q[b, h, t]) * on))
    vv = np.concatenate((v, vn))
    num, den = w[:, None] * vv, w.copy()
    unit = slice(256, 384)
    if mistake == "lost unit":
        num[unit] = 0
        den[unit] = 0
    elif mistake == "unit twice":
        num[unit] *= 2
        den[unit] *= 2
    elif mistake == "another head's unit":
        num[unit] = w[unit, None] * c.rows("v", 0, 1)[unit]
    elif mistake == "one key lost":
        num[700], den[700] = 0, 0
    elif mistake == "lost numerator":
        num[unit] = 0
    else:
        i, j = np.flatnonzero(w[:1100] == w.max())[0], np.flatnonzero(w[:1100] == w[:1100].min())[0]
        assert q[b, h, t, 0] != 0
        num[[i, j]] = w[[i, j], None] * vv[[j, i]]
    out = want[0].copy()
    ce.check_whole(out, None, want, f32)
    out[b, h, t] = num.sum(axis=0) / den.sum()
    if not f32:
        out = _bf16(out)
    if not f32 and mistake in ("one key lost", "two keys exchanged"):
        return                                           # one key of 1,100 may hide in a bf16 rounding
    with pytest.raises(AssertionError):
        ce.check_whole(out, None, want, f32)
