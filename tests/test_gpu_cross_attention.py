"""sva_cross_attention and its gradients on the GPU against oracle/cross_attention.py:
lengths of one and many tokens, grouped heads, lengths, masks and entries without keys,
keys divided among workgroups, strides, what hidden places hold."""
import math

import numpy as np
import pytest

import paper_2606_23743_amd as sva
from oracle import cross_attention as oca

from .cache_cases import bf16_normal
from .gpu_cases import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U, UB = 2.0 ** -24, 2.0 ** -8        # half a step of float32 and of bf16, relative
TINY = 2.0 ** -126                   # what is smaller may become zero: a weight, dS, a result


def _heads(x, layout):
    """The same values on the device, laid out: [B, H, N, D], token-major, or a slice of wider rows."""
    B, H, N, D = x.shape
    if layout == "plain":
        return x.cuda()
    if layout == "token":
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    y = torch.full((N, B, H + 1, D + 16), float("nan"), dtype=x.dtype, device="cuda")[:, :, 1:, 8:8 + D].permute(1, 2, 0, 3)
    return y.copy_(x)


class Case:
    def __init__(self, B, H, kv, N, M, D, hide="none", layout="plain", scale=1.0, c=0.0, seed=0, poison=True):
        say(f"[cross] B={B} H={H}/{kv} N={N} M={M} D={D} hide={hide} layout={layout} scale={scale} c={c}")
        g = np.random.default_rng(seed + B * 7 + N * 3 + M)
        q, k, v, go = (bf16_normal(g, s) for s in ((B, H, N, D), (B, kv, M, D), (B, kv, M, D), (B, H, N, D)))
        q = (q.float() * scale).to(torch.bfloat16)
        lengths = mask = None
        if "lengths" in hide:
            lengths = g.integers(0, M + 1, B)
            lengths[0] = M
            if B > 2:
                lengths[1], lengths[2] = 0, M + 5            # none; more than there are
        if "mask" in hide:
            mask = g.random((B, M)) < 0.6
            if B > 1:
                mask[-1] = False
        self.seen = oca.seen_keys(B, M, lengths, mask)
        self.c = c if c > 0 else 1.0 / math.sqrt(D)
        self.arg_c = c
        hidden = torch.from_numpy(~self.seen)[:, None, :, None].expand(B, kv, M, D)
        self.k64, self.v64 = k.double().numpy(), v.double().numpy()
        if poison:
            k[hidden], v[hidden] = float("nan"), float("inf")
        self.q64, self.go64 = q.double().numpy(), go.double().numpy()
        self.q, self.k, self.v, self.go = (_heads(t, layout) for t in (q, k, v, go))
        self.kw = dict(lengths=None if lengths is None else torch.from_numpy(lengths.astype(np.int32)).cuda(),
                       mask=None if mask is None else torch.from_numpy(mask).cuda(), softmax_scale=c)
        self.M = M

    def each(self):
        """b, h, kv head, seen keys."""
        group = self.q64.shape[1] // self.k64.shape[1]
        for b in range(self.q64.shape[0]):
            at = np.flatnonzero(self.seen[b])
            for h in range(self.q64.shape[1]):
                yield b, h, h // group, at

    def logit_error(self, b, h, kv, at):
        """A float32 sum of D exact products and a few roundings of the logit: (D + 16) U of sum |q k| c."""
        s = self.c * (np.abs(self.q64[b, h]) @ np.abs(self.k64[b, kv, at]).T)
        return U * (self.q64.shape[-1] + 16) * s.max(axis=-1, keepdims=True)

    def check_forward(self):
        out, lse = sva.cross_attention(self.q, self.k, self.v, want_lse=True, **self.kw)
        torch.cuda.synchronize()
        self.out, self.lse = oca.forward(self.q64, self.k64, self.v64, self.seen, self.c)
        got, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert out.stride() == torch.empty_like(self.q).stride()
        for b, h, kv, at in self.each():
            if len(at) == 0:
                assert not got[b, h].any() and (l[b, h] == -np.inf).all()
                continue
            e = self.logit_error(b, h, kv, at)
            p = np.exp(self.c * (self.q64[b, h] @ self.k64[b, kv, at].T) - self.lse[b, h][:, None])
            # each weight and their sum: an error of the logit on both sides, one rounding to bf16, the sums in
            # float32 (at most a fourth of the keys in a row)
            rel = 2 * (UB + 2 * e) + U * (self.M / 4 + 40)
            tol = ((rel * 1.02 * p + TINY) @ np.abs(self.v64[b, kv, at])) + UB * 1.02 * np.abs(self.out[b, h]) + TINY
            assert (np.abs(got[b, h] - self.out[b, h]) <= tol).all(), (b, h, np.abs(got[b, h] - self.out[b, h]).max())
            l_tol = 2 * e[:, 0] + U * (self.M / 4 + 48) + 4 * U * np.abs(self.lse[b, h])
            assert (np.abs(l[b, h] - self.lse[b, h]) <= l_tol).all(), (b, h, np.abs(l[b, h] - self.lse[b, h]).max())
        without, none = sva.cross_attention(self.q, self.k, self.v, **self.kw)
        assert none is None and torch.equal(without, out)      # lse does not change the result
        return self

    def check_backward(self):
        """From out rounded to bf16 and lse to float32, as the call takes them."""
        if not hasattr(self, "out"):
            self.out, self.lse = oca.forward(self.q64, self.k64, self.v64, self.seen, self.c)
        out = torch.from_numpy(self.out).to(torch.bfloat16)
        lse = torch.from_numpy(self.lse.astype(np.float32))
        o64, l64 = out.double().numpy(), lse.double().numpy()
        want = oca.backward(self.go64, self.q64, self.k64, self.v64, o64, l64, self.seen, self.c)
        out = torch.empty_like(self.q).copy_(out)
        got = sva.cross_attention_backward(self.go, self.q, self.k, self.v, out, lse.cuda(), **self.kw)
        torch.cuda.synchronize()
        for t, x in zip(got, (self.q, self.k, self.v)):
            assert t.shape == x.shape and t.dtype == torch.bfloat16
        tol = [UB * np.abs(w) for w in want]
        N, M, D = self.q64.shape[2], self.M, self.q64.shape[3]
        group = self.q64.shape[1] // self.k64.shape[1]
        for b, h, kv, at in self.each():
            if len(at) == 0:
                continue
            q, k, v, go = self.q64[b, h], self.k64[b, kv, at], self.v64[b, kv, at], self.go64[b, h]
            # a weight: the logit's error, the lse's rounding in base 2 (of both its terms), exp2's step
            e = 2 * self.logit_error(b, h, kv, at) + U * (4 * np.abs(l64[b, h])[:, None] + 8)
            p = np.exp(self.c * (q @ k.T) - l64[b, h][:, None])
            # dP and delta are float32 sums of D products
            d_err = U * (D + 8) * (np.abs(go) @ np.abs(v).T + (np.abs(go) * np.abs(o64[b, h])).sum(-1, keepdims=True))
            ds = np.abs(p * (go @ v.T - (go * o64[b, h]).sum(-1, keepdims=True)))
            # a weight below TINY may be zero: dS is then off by TINY |dP - delta|, and dS below TINY may be zero too
            lost = TINY * (1 + np.abs(go) @ np.abs(v).T + (np.abs(go) * np.abs(o64[b, h])).sum(-1, keepdims=True))
            ds_err = p * d_err * (1 + e) + ds * (e + UB + 4 * U) + lost
            # dQ and dK may be formed with what delta is without out's rounding, the sum of P dP.  For dQ that takes
            # off P K away, off being found as a float32 sum of dS and P rounded to bf16
            off = np.abs((p * (go @ v.T)).sum(-1, keepdims=True) - (go * o64[b, h]).sum(-1, keepdims=True))
            off_err = (ds_err + ds * U * (M + 40)).sum(-1, keepdims=True)
            tol[0][b, h] += self.c * ((ds_err + ds * U * (M + 40) + p * (1 + e + UB + U * (M + 40)) * (off + off_err)) @ np.abs(k))
            tol[1][b, kv, at] += self.c * ((ds_err + p * off + (ds + p * off) * U * (N * group + 300)).T @ np.abs(q))
            tol[2][b, kv, at] += (p * (e + UB + U * (N * group + 300)) + TINY).T @ np.abs(go)
        for name, a, w, t in zip(("dq", "dk", "dv"), got, want, tol):
            d = np.abs(a.double().cpu().numpy() - w)
            assert (d <= 1.02 * t + TINY).all(), (name, d.max(), (d - 1.02 * t - TINY).max())
        return self

    def check(self):
        return self.check_forward().check_backward()


HIDE = ["none", "lengths", "mask", "lengths+mask"]


@pytest.mark.parametrize("D", [64, 112, 128])
@pytest.mark.parametrize("hide", HIDE)
@pytest.mark.parametrize("N,M", [(1, 1), (1, 33), (17, 31), (64, 32), (65, 100), (130, 257)])
def test_sizes(D, hide, N, M):
    Case(4, 4, 2, N, M, D, hide).check()


@pytest.mark.parametrize("layout", ["plain", "token", "wide"])
@pytest.mark.parametrize("H,kv", [(3, 3), (5, 1), (8, 2)])
@pytest.mark.parametrize("hide", ["none", "mask"])
def test_groups_and_strides(layout, H, kv, hide):
    Case(2, H, kv, 37, 77, 128, hide, layout).check()


@pytest.mark.parametrize("D", [64, 112, 128])
@pytest.mark.parametrize("hide", HIDE)
def test_one_token_over_many_keys(D, hide):
    """Keys divided among workgroups; with a mask, lists longer than their ring in LDS."""
    Case(3, 8, 2, 1, 5000, D, hide).check()


def test_few_rows_over_one_long_state():
    Case(1, 1, 1, 3, 20011, 128, "mask").check()
    Case(1, 2, 1, 200, 4099, 64, "none").check()


def test_many_rows_over_few_keys():
    """The walk over rows divided among workgroups, and a group of heads whose tokens end inside a tile."""
    Case(1, 2, 2, 2500, 40, 128, "none").check()
    Case(2, 6, 2, 701, 130, 112, "mask").check()


def test_rows_of_32_a_wave():
    """Enough rows for the wide form, and more key tiles than parts."""
    Case(2, 40, 40, 900, 50, 64, "lengths").check()
    Case(1, 64, 64, 1100, 20, 128, "none").check()
    Case(1, 66, 66, 1030, 20, 112, "mask").check()


@pytest.mark.parametrize("hide", HIDE)
def test_rows_of_32_a_wave_over_divided_keys(hide):
    """Parts without a key where lengths are short, joined by a wave (few parts) or four."""
    Case(3, 3, 1, 600, 3500, 112, hide).check()
    Case(1, 1, 1, 1500, 2600, 64, hide, "token").check()


@pytest.mark.parametrize("hide", ["none", "mask"])
def test_large_logits_and_rising_ones(hide):
    """Logits of hundreds, the largest in the last key: the reference has to follow."""
    case = Case(2, 4, 2, 40, 300, 64, hide, scale=40.0, poison=False)
    case.check()
    for c in (1e-3, 2.0):
        Case(2, 2, 2, 20, 90, 128, hide, c=c).check()
    rising = Case(1, 2, 2, 33, 400, 64, "none")
    grow = np.linspace(0.1, 60.0, 400)[None, None, :, None]
    k = torch.from_numpy(np.abs(rising.k64) * grow).to(torch.bfloat16)
    q = torch.from_numpy(np.abs(rising.q64)).to(torch.bfloat16)
    rising.k64, rising.q64, rising.k, rising.q = k.double().numpy(), q.double().numpy(), k.cuda(), q.cuda()
    rising.check()


def test_infinite_and_bad_inputs_stay_in_their_rows():
    case = Case(1, 2, 2, 20, 50, 64, "none")
    q = case.q.clone()
    q[0, 0, 3] = float("nan")
    out, lse = sva.cross_attention(q, case.k, case.v, want_lse=True)
    assert torch.isnan(out[0, 0, 3]).all() and torch.isnan(lse[0, 0, 3])
    want, _ = sva.cross_attention(case.q, case.k, case.v)
    keep = [i for i in range(20) if i != 3]
    assert torch.equal(out[0, 0, keep], want[0, 0, keep]) and torch.equal(out[0, 1], want[0, 1])
    # keys far below every other weigh nothing, whatever the sign of their logit
    k = case.k.clone()
    k[0, :, 7:] = 0.0
    k[0, :, 7:, 0] = torch.finfo(torch.bfloat16).min / 4
    q = case.q.abs() + 0.1
    out, lse = sva.cross_attention(q, k, case.v, want_lse=True)
    want, l = sva.cross_attention(q, k[:, :, :7], case.v[:, :, :7], want_lse=True)
    assert torch.equal(out, want) and torch.equal(lse, l)


def test_lengths_are_clamped_and_a_mask_may_be_shared():
    case = Case(3, 2, 1, 9, 70, 128, "none")
    out, _ = sva.cross_attention(case.q, case.k, case.v, lengths=torch.tensor([-4, 1000, 70], dtype=torch.int32, device="cuda"))
    want, _ = sva.cross_attention(case.q, case.k, case.v)
    assert not out[0].any() and torch.equal(out[1:], want[1:])
    mask = torch.rand(70, device="cuda") < 0.5
    one, _ = sva.cross_attention(case.q, case.k, case.v, mask=mask)
    all_, _ = sva.cross_attention(case.q, case.k, case.v, mask=mask.expand(3, 70).contiguous().to(torch.uint8) * 7)
    assert torch.equal(one, all_)


def test_states_past_32_bits_and_inputs_that_repeat_themselves():
    big = torch.empty((1 << 32) + (1 << 21), dtype=torch.bfloat16, device="cuda")
    data = torch.randn((2, 1, 3, 128), device="cuda").to(torch.bfloat16)
    far = big.as_strided((2, 1, 3, 128), (1 << 31, 1, 1 << 30, 1))
    far[0].copy_(data[0])
    far[1, :, 1:].copy_(data[1, :, 1:])
    data[1, :, 0] = far[1, :, 0]                          # one place with entry 0's last
    q = torch.randn((2, 2, 5, 128), device="cuda").to(torch.bfloat16)
    for mask in (None, torch.tensor([[True, False, True], [True, True, True]], device="cuda")):
        want = sva.cross_attention(q, data, data, mask=mask, want_lse=True)
        got = sva.cross_attention(q, far, far, mask=mask, want_lse=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        gw = sva.cross_attention_backward(q, q, data, data, *want, mask=mask)
        gg = sva.cross_attention_backward(q, q, far, far, *want, mask=mask, dk=torch.empty_like(data), dv=torch.empty_like(data))
        assert all(torch.equal(a, b) for a, b in zip(gg, gw))
    del big, far
    same = q[:, :1, :1].expand(2, 2, 5, 128)
    out, _ = sva.cross_attention(same, data[:1].expand(2, 1, 3, 128), data[:1].expand(2, 1, 3, 128),
                                 out=torch.empty_like(q))
    full, _ = sva.cross_attention(same.contiguous(), data[:1].repeat(2, 1, 1, 1), data[:1].repeat(2, 1, 1, 1))
    assert torch.equal(out, full)


@pytest.mark.parametrize("N,M,D", [(64, 96, 128), (24, 1600, 64)])        # keys in one part and in several
def test_gradients_do_not_carry_the_rounding_of_out(N, M, D):
    """Rows with one large weight: delta from out as rounded to bf16 would be further off than dS itself."""
    c = Case(1, 2, 1, N, M, D, scale=5.0, seed=3)
    out, lse = sva.cross_attention(c.q, c.k, c.v, want_lse=True)
    dq, dk, _ = (x.double().cpu().numpy() for x in sva.cross_attention_backward(c.go, c.q, c.k, c.v, out, lse))
    o64, l64 = oca.forward(c.q64, c.k64, c.v64, c.seen, c.c)
    want = oca.backward(c.go64, c.q64, c.k64, c.v64, o64, l64, c.seen, c.c)
    given = out.double().cpu().numpy()
    tol_k, past = UB * np.abs(want[1]), 0
    for b, h, kv, at in c.each():
        q, k, v, go = c.q64[b, h], c.k64[b, kv, at], c.v64[b, kv, at], c.go64[b, h]
        # a weight: errors of the logit here and in lse, whose sum and rounding, exp2's step
        e = 4 * c.logit_error(b, h, kv, at) + U * (M / 4 + 56 + 8 * np.abs(l64[b, h])[:, None])
        p, dp = np.exp(c.c * (q @ k.T) - l64[b, h][:, None]), go @ v.T
        delta = (p * dp).sum(-1, keepdims=True)
        off = np.abs((go * given[b, h]).sum(-1, keepdims=True) - delta)     # what out's rounding takes from it
        d_err = U * (D + 8) * (np.abs(go) @ np.abs(v).T + (np.abs(go) * np.abs(given[b, h])).sum(-1, keepdims=True))
        ds = p * (np.abs(dp - delta) + off)                                 # as large as it may be when it is rounded
        ds_f32 = p * d_err * (1 + e) + ds * (e + U * (M + 44)) + TINY * (1 + np.abs(dp) + np.abs(delta))
        e_err = ds_f32.sum(-1, keepdims=True)                               # e is a sum of dS in float32
        pk = p @ np.abs(k)
        tol = UB * np.abs(want[0][b, h]) + c.c * ((ds_f32 + ds * UB) @ np.abs(k) + pk * (off * (e.max() + UB + U * (M + 40)) + e_err))
        d = np.abs(dq[b, h] - want[0][b, h])
        assert (d <= 1.02 * tol + TINY).all(), (h, d.max(), (d - 1.02 * tol).max())
        past += (c.c * off * np.abs(p @ k) > 2 * tol).sum()
        d_k = p * (dp - delta)
        tol_k[b, kv, at] += c.c * ((ds_f32 + p * e_err + np.abs(d_k) * (UB + U * (4 * N + 300)) + p * U * 8 * np.abs(delta)).T @ np.abs(q))
    assert past > 0                                                         # without the correction these would fail
    d = np.abs(dk - want[1])
    assert (d <= 1.02 * tol_k + TINY).all(), (d.max(), (d - 1.02 * tol_k).max())


def test_gradient_against_differences():
    """Central differences of the 64-bit forward at bf16 inputs; the kernels' own roundings are what is allowed."""
    case = Case(1, 2, 1, 3, 6, 64, "none", seed=3)
    out, lse = sva.cross_attention(case.q, case.k, case.v, want_lse=True)
    grads = sva.cross_attention_backward(case.go, case.q, case.k, case.v, out, lse)
    h = 1e-5
    for name, x, d in zip("qkv", (case.q64, case.k64, case.v64), grads):
        d = d.double().cpu().numpy()
        # dS of this case is below 20, rounded with its weight and delta: 4 UB of sums of six such products
        for at in list(np.ndindex(*x.shape))[::37]:
            keep = x[at]
            ends = []
            for s in (h, -h):
                x[at] = keep + s
                ends.append((oca.forward(case.q64, case.k64, case.v64, case.seen, case.c)[0] * case.go64).sum())
            x[at] = keep
            assert abs(d[at] - (ends[0] - ends[1]) / (2 * h)) <= 4 * UB * 6 * 20 * (case.c if name != "v" else 0.1), (name, at)


def test_outputs_given_and_hidden_rows_of_the_gradients_written():
    case = Case(2, 4, 2, 50, 90, 128, "mask")
    out, lse = torch.full_like(case.q, 7.0), torch.full((2, 4, 50), 7.0, device="cuda")
    a, l = sva.cross_attention(case.q, case.k, case.v, out=out, lse=lse, **case.kw)
    assert a is out and l is lse and not out[1].any() and torch.isinf(lse[1]).all()
    dk, dv = torch.full_like(case.k, 7.0), torch.full_like(case.v, 7.0)
    ws = torch.empty(sva.cross_attention_workspace(2, 4, 2, 50, 90, 128, masked=True, backward=True), dtype=torch.uint8,
                     device="cuda")
    ws.fill_(255)                                          # contents on entry do not matter
    dq, _, _ = sva.cross_attention_backward(case.go, case.q, case.k, case.v, out, lse, dk=dk, dv=dv, workspace=ws, **case.kw)
    hidden = torch.from_numpy(~case.seen).cuda()
    assert not dk.transpose(1, 2)[hidden].any() and not dv.transpose(1, 2)[hidden].any() and not dq[1].any()
    assert dk.transpose(1, 2)[~hidden].any()


def test_same_bits_twice_and_on_a_side_stream():
    case = Case(2, 8, 4, 300, 700, 128, "lengths+mask")

    def step(s):
        o, l = sva.cross_attention(case.q, case.k, case.v, want_lse=True, stream=s, **case.kw)
        return [o, l, *sva.cross_attention_backward(case.go, case.q, case.k, case.v, o, l, stream=s, **case.kw)]

    want = step(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(want, got, step(None)):
        assert torch.equal(a, b) and torch.equal(a, c)
