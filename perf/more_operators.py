"""Performance cases of what stands around self-attention in a denoiser's layer, through the
package's public entry points.

Kinds of case
  norm   layer_norm, and layer_norm_backward where the case trains: weight and bias one row
         for all tokens, or one row per batch entry added to one (adaptive norm)
  axes   rotary_axes_plan -> rotary_axes on Q and K: positions on several axes (time, height,
         width), whole or fractional; forward or gradient
  cross  cross_attention of N tokens to M states of an encoder, with lengths or a mask;
         where the case trains, cross_attention_backward after it

Tensors of heads are [B, H, N, D]; where a case says token_major the memory behind them is
[B, N, H, D], as a projection leaves it.
"""
import math

import torch

own = False

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
_TYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # one token of eight running sequences, adaptive: launch latency
        dict(name="norm_step", kind="norm", batch=8, tokens=1, channels=4096, dtype="bf16", per_entry=True, train=False),
        # the tokens of a 22B-class layer, adaptive, for sampling
        dict(name="norm_long", kind="norm", batch=1, tokens=63240, channels=4096, dtype="bf16", per_entry=True, train=False),
        # a guidance pair of a 2B-class layer, adaptive, one training step
        dict(name="norm_train", kind="norm", batch=2, tokens=32760, channels=2240, dtype="bf16", per_entry=True, train=True),
        # float32 rows of odd length with a shared weight and bias
        dict(name="norm_train_odd", kind="norm", batch=3, tokens=7801, channels=1001, dtype="f32", per_entry=False,
             train=True),
        # one frame of a guidance pair, streamed: small
        dict(name="axes_frame", kind="axes", batch=2, heads=20, kv_heads=20, tokens=1560, dim=112, sections="20,18,18",
             layout="interleaved", fractional=False, dtype="bf16", backward=False, token_major=True),
        # gradients of a 22B-class layer's Q and K, time in seconds (fractional)
        dict(name="axes_train", kind="axes", batch=1, heads=32, kv_heads=8, tokens=63240, dim=128, sections="16,24,24",
             layout="half", fractional=True, dtype="bf16", backward=True, token_major=True),
        # one token of eight sequences over a prompt's states, grouped heads: latency
        dict(name="cross_step", kind="cross", batch=8, heads=32, kv_heads=8, queries=1, keys=1560, dim=128, hide="lengths",
             lse=False, train=False, token_major=True),
        # seven tokens over two long encoded videos: the keys are the work
        dict(name="cross_step_long", kind="cross", batch=2, heads=48, kv_heads=8, queries=7, keys=111600, dim=128, hide="none",
             lse=True, train=False, token_major=False),
        # a guidance pair over its padded prompts, with holes in the mask
        dict(name="cross_text", kind="cross", batch=2, heads=20, kv_heads=20, queries=32760, keys=512, dim=112, hide="mask",
             lse=False, train=False, token_major=True),
        # a small training batch of odd sizes, prompts of unequal length, one of them empty
        dict(name="cross_train_odd", kind="cross", batch=5, heads=8, kv_heads=4, queries=1001, keys=77, dim=64, hide="lengths",
             lse=True, train=True, token_major=True),
        # a 22B-class layer's tokens over a prompt, for sampling
        dict(name="cross_long", kind="cross", batch=1, heads=32, kv_heads=32, queries=63240, keys=512, dim=128, hide="none",
             lse=False, train=False, token_major=True),
        # the same, one training step
        dict(name="cross_train", kind="cross", batch=1, heads=32, kv_heads=32, queries=63240, keys=512, dim=128, hide="none",
             lse=True, train=True, token_major=True),
    ]


_MOST = {"norm": (1.18e9, 1e12), "axes": (1.3e9, 1e12), "cross": (2.6e9, 1.86e12)}


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.5 / hi))))

    while True:
        kind = rng.choice(["norm", "norm", "axes", "cross", "cross", "cross"])
        batch = rng.choice([1, 1, 2, 3, 8, 31])
        dim = rng.choice([64, 112, 128, 128])
        kv = log_int(1, 32)
        if kind == "norm":
            channels = rng.choice([log_int(8, 8192), 8 * log_int(1, 1024), 8 * log_int(64, 1024)])
            c = dict(kind=kind, batch=batch, tokens=log_int(1, 63240), channels=channels, dtype=rng.choice(["bf16", "bf16", "f32"]),
                     per_entry=rng.random() < 0.5, train=rng.random() < 0.5)
        elif kind == "axes":
            axes = rng.choice([2, 3, 3, 3, 4])
            pairs, cuts = dim // 2, sorted(rng.sample(range(1, dim // 2), axes - 1))
            if rng.random() < 0.2:
                pairs -= 8                       # the head's last channels are not turned
                cuts = sorted(rng.sample(range(1, pairs), axes - 1))
            sections = [b - a for a, b in zip([0] + cuts, cuts + [pairs])]
            c = dict(kind=kind, batch=batch, heads=kv * rng.choice([1, 1, 2, 4, 8]), kv_heads=kv, tokens=log_int(1, 63240),
                     dim=dim, sections=",".join(map(str, sections)), layout=rng.choice(["half", "interleaved"]),
                     fractional=rng.random() < 0.4, dtype=rng.choice(["bf16", "bf16", "f32"]),
                     backward=rng.random() < 0.4, token_major=rng.random() < 0.6)
        else:
            train = rng.random() < 0.45
            c = dict(kind=kind, batch=batch, heads=kv * rng.choice([1, 1, 1, 2, 4, 5, 8]), kv_heads=kv,
                     queries=log_int(1, 63240), keys=log_int(2 if train else 1, rng.choice([1024, 111600])), dim=dim,
                     hide=rng.choice(["none", "lengths", "lengths", "mask"]), lse=train or rng.random() < 0.4, train=train,
                     token_major=rng.random() < 0.6)
        full = work({**c, "hide": "none"}) if kind == "cross" else work(c)
        if full["bytes"] > _MOST[kind][0] or full["flops"] > _MOST[kind][1]:
            continue
        # the plain form holds every logit, and every key and value in 32 bits
        if kind != "cross" or max(batch * c["heads"] * c["queries"] * c["keys"], batch * kv * c["keys"] * dim) <= 1.04e9:
            return c


# ------------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, batch, heads, tokens, dim, dtype, token_major, scale=1.0):
    """N(0, scale^2) values [B, H, N, D], the memory behind them [B, N, H, D] if token_major."""
    shape = (batch, tokens, heads, dim) if token_major else (batch, heads, tokens, dim)
    x = torch.randn(shape, generator=g, device="cuda", dtype=F32).mul_(scale).to(dtype)
    return x.transpose(1, 2) if token_major else x


def _hidden_states(case, g):
    """Rows of a residual stream: unequal sizes, a mean of their own, a few channels far larger."""
    b, n, c = case["batch"], case["tokens"], case["channels"]
    x = torch.randn((b, n, c), generator=g, device="cuda", dtype=F32)
    gain = torch.ones(c, device="cuda", dtype=F32)
    gain[torch.randint(0, c, (max(1, c // 256),), generator=g, device="cuda")] = 12.0
    size = torch.exp(0.5 * torch.randn((b, n, 1), generator=g, device="cuda", dtype=F32))
    return x.mul_(gain).add_(torch.randn((b, n, 1), generator=g, device="cuda", dtype=F32)).mul_(size).to(_TYPES[case["dtype"]])


def _positions(case, g):
    """[B, N, axes]: tokens in raster order over a video's grid, from a frame of its own on; fractional:
    time in seconds at 24 frames of 4 a step, height and width from their middle."""
    n, axes = case["tokens"], len(case["sections"].split(","))
    side = max(1, round((n / 16) ** 0.5))
    at = torch.arange(n, device="cuda")
    grid = [at // (side * side), at // side % side, at % side, at % 7][:axes]
    p = torch.stack(grid, dim=-1).expand(case["batch"], n, axes).clone()
    p[..., 0] += torch.randint(0, 200, (case["batch"], 1), generator=g, device="cuda")
    if not case["fractional"]:
        return p.to(torch.int32)
    scale = torch.tensor([4.0 / 24.0, 1.0, 1.0, 1.0][:axes], dtype=F64, device="cuda")
    first = torch.tensor([0.0, side / 2.0, side / 2.0, 0.0][:axes], dtype=F64, device="cuda")
    return (p.double() * scale - first).float()


def _hidden_keys(case, g):
    """(int32 [B] or None, bool [B, M] or None): the first entry has all its keys, the others
    any number of them, the last one of five or more none."""
    b, m = case["batch"], case["keys"]
    n = torch.randint(1, m + 1, (b,), generator=g, device="cuda")
    n[0] = m
    if b >= 5:
        n[-1] = 0
    if case["hide"] == "lengths":
        return n.to(torch.int32), None
    if case["hide"] == "mask":
        holes = torch.rand((b, m), generator=g, device="cuda") < 0.1
        return None, (torch.arange(m, device="cuda") < n[:, None]) & ~holes
    return None, None


def prepare(case, seed):
    g = _generator(seed)
    st = {"case": case}
    if case["kind"] == "norm":
        b, c = case["batch"], case["channels"]
        rows = (b, c) if case["per_entry"] else (c,)
        st["x"] = _hidden_states(case, g)
        st["weight"] = torch.randn(rows, generator=g, device="cuda", dtype=F32).mul_(0.3)
        if not case["per_entry"]:
            st["weight"] += 1.0
        st["bias"] = torch.randn(rows, generator=g, device="cuda", dtype=F32).mul_(0.3)
        if case["train"]:
            st["dy"] = torch.randn(st["x"].shape, generator=g, device="cuda", dtype=F32).to(st["x"].dtype)
        return st
    b, h, kv, dim, major = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["token_major"]
    if case["kind"] == "axes":
        kind = _TYPES[case["dtype"]]
        st["q"] = _normal(g, b, h, case["tokens"], dim, kind, major)
        st["k"] = _normal(g, b, kv, case["tokens"], dim, kind, major)
        st["positions"] = _positions(case, g)
        st["freq"], st["axis"] = _ladders(case)
        if own:
            import paper_2606_23743_amd as sva
            st["plan"] = sva.rotary_axes_plan(dim, [int(n) for n in case["sections"].split(",")], layout=case["layout"])
        return st
    n, m = case["queries"], case["keys"]
    st["q"] = _normal(g, b, h, n, dim, BF16, major, 1.5)
    st["k"] = _normal(g, b, kv, m, dim, BF16, major)
    st["v"] = _normal(g, b, kv, m, dim, BF16, major)
    st["k"][:, :, 0] *= 2.0                      # a prompt's first state draws more
    st["lengths"], st["mask"] = _hidden_keys(case, g)
    if case["train"]:
        st["dout"] = _normal(g, b, h, n, dim, BF16, major)
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    if not own:
        return {"norm": _norm_plain, "axes": _axes_plain, "cross": _cross_plain}[case["kind"]](st)
    import paper_2606_23743_amd as sva
    if case["kind"] == "norm":
        adaptive = case["per_entry"]
        if not case["train"]:
            return sva.layer_norm(st["x"], st["weight"], st["bias"], eps=_EPS, unit_offset=adaptive)[0]
        y, mean, rstd = sva.layer_norm(st["x"], st["weight"], st["bias"], eps=_EPS, unit_offset=adaptive, want_stats=True)
        return (y, *sva.layer_norm_backward(st["dy"], st["x"], mean, rstd, st["weight"], unit_offset=adaptive))
    if case["kind"] == "axes":
        return sva.rotary_axes(st["plan"], st["positions"], st["q"], st["k"], backward=case["backward"])
    hide = dict(lengths=st["lengths"], mask=st["mask"])
    out, lse = sva.cross_attention(st["q"], st["k"], st["v"], want_lse=case["lse"], **hide)
    if not case["train"]:
        return (out, lse) if case["lse"] else out
    return (out, lse, *sva.cross_attention_backward(st["dout"], st["q"], st["k"], st["v"], out, lse, **hide))


_EPS = 1e-6


def _norm_plain(st):
    case = st["case"]
    x = st["x"].float()
    w, bias = (r[:, None] if case["per_entry"] else r for r in (st["weight"], st["bias"]))
    w = 1.0 + w if case["per_entry"] else w
    d = x - x.mean(dim=-1, keepdim=True)
    rstd = (d * d).mean(dim=-1, keepdim=True).add(_EPS).rsqrt()
    xhat = d * rstd
    y = (xhat * w + bias).to(st["x"].dtype)
    if not case["train"]:
        return y
    dy = st["dy"].float()
    over = (1,) if case["per_entry"] else (0, 1)
    gr = dy * w
    dx = rstd * (gr - gr.mean(dim=-1, keepdim=True) - xhat * (gr * xhat).mean(dim=-1, keepdim=True))
    return y, dx.to(y.dtype), (dy * xhat).sum(dim=over), dy.sum(dim=over)


def _ladders(case):
    """Radians per unit of each pair's axis, base^(-i/n) in an axis of n pairs, and the axis of each pair."""
    n = torch.tensor([int(s) for s in case["sections"].split(",")], device="cuda")
    axis = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n)
    index = torch.arange(axis.numel(), device="cuda") - (n.cumsum(0) - n)[axis]
    return 10000.0 ** (-index.double() / n[axis].double()), axis


def _axes_plain(st):
    case, pairs = st["case"], st["axis"].numel()
    angle = st["positions"].double()[..., st["axis"]] * st["freq"]        # far positions need 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    sin = -sin if case["backward"] else sin

    def turn(x):
        y = x.float()
        if case["layout"] == "half":
            a, b = y[..., :pairs], y[..., pairs:2 * pairs]
            t = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
        else:
            a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
            t = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
        return torch.cat((t, y[..., 2 * pairs:]), dim=-1).to(x.dtype)

    return turn(st["q"]), turn(st["k"])


def _seen(st):
    """bool [B, M] or None."""
    if st["lengths"] is not None:
        return torch.arange(st["case"]["keys"], device="cuda") < st["lengths"][:, None]
    return st["mask"]


def _cross_plain(st):
    case = st["case"]
    b, h, kv, n, m, dim = (case[x] for x in ("batch", "heads", "kv_heads", "queries", "keys", "dim"))
    scale, seen = 1.0 / math.sqrt(dim), _seen(st)
    rows = (b, kv, h // kv * n, dim)                                        # the queries of a group share their keys
    q = st["q"].float().reshape(rows)
    k, v = st["k"].float().contiguous(), st["v"].float().contiguous()
    s = (q * scale) @ k.transpose(2, 3)
    if seen is not None:
        s = torch.where(seen[:, None, None], s, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    del s
    total = p.sum(dim=-1, keepdim=True)
    out32 = torch.where(total > 0, (p @ v) / total, 0.0)
    out = out32.to(BF16).reshape(b, h, n, dim)
    lse = (top + total.log()).reshape(b, h, n)
    if not case["train"]:
        return (out, lse) if case["lse"] else out
    p = p / torch.where(total > 0, total, 1.0)
    dout = st["dout"].float().reshape(rows)
    dv = p.transpose(2, 3) @ dout
    delta = (dout * out32).sum(dim=-1, keepdim=True)
    ds = p.mul_((dout @ v.transpose(2, 3)).sub_(delta))
    dq = (ds @ k) * scale
    dk = (ds.transpose(2, 3) @ q) * scale
    return out, lse, dq.to(BF16).reshape(b, h, n, dim), dk.to(BF16), dv.to(BF16)


# ------------------------------------------------------- work and definitions

def work(case):
    b = case["batch"]
    if case["kind"] == "norm":
        item, count = 2 if case["dtype"] == "bf16" else 4, b * case["tokens"] * case["channels"]
        rows = case["channels"] * (b if case["per_entry"] else 1) * 4
        if case["train"]:                        # x, dy -> y, dx, and both rows with their gradients
            return {"bytes": 4 * count * item + 4 * rows, "flops": 22 * count}
        return {"bytes": 2 * count * item + 2 * rows, "flops": 8 * count}
    dim, h, kv = case["dim"], case["heads"], case["kv_heads"]
    if case["kind"] == "axes":
        item, n, axes = 2 if case["dtype"] == "bf16" else 4, b * case["tokens"], len(case["sections"].split(","))
        turned = 2 * sum(int(s) for s in case["sections"].split(","))
        return {"bytes": 2 * n * (h + kv) * dim * item + 4 * axes * n, "flops": 3 * n * (h + kv) * turned}
    # keys are hidden as the inputs are drawn: their mean over seeds
    n, m = case["queries"], case["keys"]
    mean = (m + 1) / 2.0
    seen = b * m if case["hide"] == "none" else m + (b - 1 - (b >= 5)) * mean
    seen = 0.9 * seen if case["hide"] == "mask" else seen
    rows, states = b * h * n * dim, kv * seen * dim
    out = {"bytes": 2 * (2 * rows + 2 * states) + (4 * b * h * n if case["lse"] else 0), "flops": 4 * h * n * seen * dim}
    if case["train"]:                            # dout -> dq, dk, dv
        out = {"bytes": out["bytes"] + 2 * (2 * rows + 2 * kv * b * m * dim), "flops": out["flops"] + 10 * h * n * seen * dim}
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _norm_exact, "axes": _axes_exact, "cross": _cross_exact}[case["kind"]](st)


def _norm_exact(st):
    """Gradients from the derivative of y_j = w_j (x_j - mu) / s + b_j, entry by entry."""
    case, c = st["case"], st["case"]["channels"]
    ys, dxs, dws, dbs = [], [], [], []
    for i in range(case["batch"]):
        x = st["x"][i].double()
        w = st["weight"][i].double() + 1.0 if case["per_entry"] else st["weight"].double()
        shift = (st["bias"][i] if case["per_entry"] else st["bias"]).double()
        mu = x.sum(dim=1, keepdim=True) / c
        s = torch.sqrt(torch.square(x - mu).sum(dim=1, keepdim=True) / c + _EPS)
        z = (x - mu) / s
        ys.append(torch.addcmul(shift, z, w))
        if case["train"]:
            dy = st["dy"][i].double()
            a = dy * w / s
            along = (a * z).sum(dim=1, keepdim=True) / c
            dxs.append(a - a.sum(dim=1, keepdim=True) / c - z * along)
            dws.append((dy * z).sum(dim=0))
            dbs.append(dy.sum(dim=0))
    y = torch.stack(ys)
    if not case["train"]:
        return y
    dw, db = torch.stack(dws), torch.stack(dbs)
    return (y, torch.stack(dxs), dw, db) if case["per_entry"] else (y, torch.stack(dxs), dw.sum(dim=0), db.sum(dim=0))


def _axes_exact(st):
    """Pair i of a token, as a complex number, times exp(+-i angle)."""
    case = st["case"]
    turns, at = [], 0
    for axis, count in enumerate(int(s) for s in case["sections"].split(",")):
        f = torch.exp(torch.arange(count, dtype=F64, device="cuda") * (-math.log(10000.0) / count))
        turns.append(st["positions"][..., axis:axis + 1].double() * f)
        at += count
    angle = torch.cat(turns, dim=-1).unsqueeze(1)
    z = torch.polar(torch.ones_like(angle), -angle if case["backward"] else angle)

    def turn(x):
        y = x.double().clone()
        first, second = (slice(0, at), slice(at, 2 * at)) if case["layout"] == "half" else (slice(0, 2 * at, 2), slice(1, 2 * at, 2))
        w = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * z
        y[..., first], y[..., second] = w.real, w.imag
        return y

    return turn(st["q"]), turn(st["k"])


def _cross_exact(st):
    """Entry by entry and head by head over the visible keys alone."""
    case = st["case"]
    b, h, kv, n, m, dim = (case[x] for x in ("batch", "heads", "kv_heads", "queries", "keys", "dim"))
    seen = _seen(st)
    out = torch.zeros((b, h, n, dim), dtype=F64, device="cuda")
    lse = torch.full((b, h, n), -math.inf, dtype=F64, device="cuda")
    dq, dk, dv = torch.zeros_like(out), *(torch.zeros((b, kv, m, dim), dtype=F64, device="cuda") for _ in range(2))
    for i in range(b):
        at = torch.arange(m, device="cuda") if seen is None else seen[i].nonzero()[:, 0]
        if at.numel() == 0:
            continue
        for j in range(h):
            c = j // (h // kv)
            k, v, q = st["k"][i, c, at].double(), st["v"][i, c, at].double(), st["q"][i, j].double()
            s = torch.matmul(q, k.t().contiguous()) * dim ** -0.5
            lse[i, j] = torch.logsumexp(s, dim=-1)
            p = torch.softmax(s, dim=-1)
            out[i, j] = torch.matmul(p, v)
            if case["train"]:
                g = st["dout"][i, j].double()
                dv[i, c, at] += torch.matmul(p.t().contiguous(), g)
                dp = torch.matmul(g, v.t().contiguous())
                ds = p * (dp - (p * dp).sum(dim=-1, keepdim=True)) * dim ** -0.5
                dq[i, j] = torch.matmul(ds, k)
                dk[i, c, at] += torch.matmul(ds.t().contiguous(), q)
    if not case["train"]:
        return (out, lse) if case["lse"] else out
    return out, lse, dq, dk, dv
