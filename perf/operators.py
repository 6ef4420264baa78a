"""Performance cases of the key/value cache operators and the rotary positions that
feed them, through the package's public entry points.

Kinds of case
  rotary  rotary_plan -> rotary on Q and K (one token of a step, a prompt, a gradient)
  write   cache_write: K and V quantised into the pages of a cache
  read    cache_read: tokens of a cache back as K and V in [B, H, N, D]
  attend  cache_attention: one or several drafted tokens over a paged cache

Tensors are [B, H, N, D]; where a case says token_major the memory behind them is
[B, N, H, D], as a projection leaves it.  A cache is {k, v: [pages, kv_heads, page, D],
k_scale, v_scale: float32 [pages, kv_heads, page]} (bf16: no scales); its codes are
e4m3 bytes (uint8) or int8, its scales one per token and head.
"""
import math

import numpy as np
import torch

own = False

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
_TYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # one token of eight running sequences, grouped heads: launch latency
        dict(name="rotary_step", kind="rotary", batch=8, heads=32, kv_heads=8, tokens=1, dim=128, rot=128,
             layout="half", scaling="none", factor=1.0, orig=0, base=10000.0, dtype="bf16", backward=False,
             token_major=True, start=2000),
        # a long prompt past its training length: half of each head turned, by-parts scaling
        dict(name="rotary_long", kind="rotary", batch=1, heads=32, kv_heads=8, tokens=63240, dim=128, rot=64,
             layout="half", scaling="yarn", factor=8.0, orig=8192, base=500000.0, dtype="bf16", backward=False,
             token_major=True, start=0),
        # gradients of Q and K in float32, interleaved pairs, odd token count, positions interpolated
        dict(name="rotary_grad", kind="rotary", batch=2, heads=20, kv_heads=20, tokens=7801, dim=112, rot=112,
             layout="interleaved", scaling="linear", factor=4.0, orig=0, base=10000.0, dtype="f32", backward=True,
             token_major=False, start=0),
        # one token of 64 sequences into an 8-bit cache
        dict(name="write_step", kind="write", batch=64, kv_heads=8, tokens=1, dim=128, page=64, fmt="e4m3",
             dtype="bf16", token_major=True),
        # a guidance pair's prompt, 112 channels, int8, small pages
        dict(name="write_prompt", kind="write", batch=2, kv_heads=20, tokens=16380, dim=112, page=16, fmt="int8",
             dtype="bf16", token_major=True),
        # K and V of 111,600 tokens (the 64B-class layer's sequence, grouped heads) into e4m3
        dict(name="write_long", kind="write", batch=1, kv_heads=8, tokens=111600, dim=128, page=128, fmt="e4m3",
             dtype="bf16", token_major=False),
        # the same sequence read back for the attention over whole sequences
        dict(name="read_long", kind="read", batch=1, kv_heads=8, tokens=111600, dim=128, page=128, fmt="e4m3",
             dtype="bf16"),
        # a prefix of odd length, int8, as float32
        dict(name="read_prefix", kind="read", batch=2, kv_heads=20, tokens=7801, dim=112, page=16, fmt="int8",
             dtype="f32"),
        # one token of four short sequences over a bf16 cache: latency
        dict(name="attend_step", kind="attend", batch=4, heads=32, kv_heads=8, drafts=1, dim=128, page=16,
             fmt="bf16", max_len=1560, ragged=True, lse=False, counts=False, out="bf16", token_major=True),
        # a serving batch of ragged lengths, one token each, e4m3
        dict(name="attend_batch", kind="attend", batch=48, heads=32, kv_heads=8, drafts=1, dim=128, page=64,
             fmt="e4m3", max_len=32760, ragged=True, lse=False, counts=False, out="bf16", token_major=True),
        # trees of up to 48 drafted tokens over long int8 caches, fewer drafts in some sequences
        dict(name="attend_tree", kind="attend", batch=8, heads=24, kv_heads=6, drafts=48, dim=128, page=64,
             fmt="int8", max_len=75600, ragged=True, lse=True, counts=True, out="bf16", token_major=True),
        # two very long sequences, seven drafted tokens, bf16 cache
        dict(name="attend_long", kind="attend", batch=2, heads=48, kv_heads=8, drafts=7, dim=128, page=128,
             fmt="bf16", max_len=223200, ragged=False, lse=True, counts=False, out="f32", token_major=True),
    ]


_MOST_BYTES = {"rotary": 1.3e9, "write": 6.8e8, "read": 6.8e8, "attend": 1.8e9}
_MOST_FLOPS = 3.2e11


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.5 / hi))))

    while True:
        kind = rng.choice(["rotary", "rotary", "write", "write", "read", "attend", "attend", "attend", "attend"])
        dim = rng.choice([64, 112, 128, 128])
        kv = log_int(1, 32)
        if kind == "rotary":
            layout = rng.choice(["half", "interleaved"])
            scaling = rng.choice(["none", "none", "linear", "ntk", "yarn"])
            c = dict(kind=kind, batch=rng.choice([1, 1, 2, 3, 8, 31, 64]), heads=kv * rng.choice([1, 1, 2, 4, 5, 8]),
                     kv_heads=kv, tokens=log_int(1, 63240), dim=dim,
                     rot=rng.choice([dim, dim, dim // 2, 2 * rng.randint(4, dim // 2)]), layout=layout,
                     scaling=scaling, factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 32.0), 2),
                     orig=rng.choice([4096, 8192, 32768]) if scaling == "yarn" else 0,
                     base=rng.choice([10000.0, 500000.0, 1000000.0]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     backward=rng.random() < 0.35, token_major=rng.random() < 0.6,
                     start=rng.choice([0, log_int(1, 1000000)]))
        elif kind in ("write", "read"):
            c = dict(kind=kind, batch=rng.choice([1, 1, 2, 3, 8, 31, 64]), kv_heads=kv, tokens=log_int(1, 111600),
                     dim=dim, page=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["bf16", "e4m3", "e4m3", "int8", "int8"]),
                     dtype=rng.choice(["bf16", "bf16", "f32"]))
            if kind == "write":
                c.update(token_major=rng.random() < 0.6)
        else:
            c = dict(kind=kind, batch=log_int(1, 64), heads=kv * rng.choice([1, 2, 4, 5, 6, 8]), kv_heads=kv,
                     drafts=rng.choice([1, 1, 1, log_int(2, 64), log_int(2, 64)]), dim=dim,
                     page=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["bf16", "e4m3", "e4m3", "int8"]),
                     max_len=log_int(1, 223200), ragged=rng.random() < 0.6, lse=rng.random() < 0.5,
                     counts=rng.random() < 0.3, out=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                     token_major=rng.random() < 0.6)
        full = work({**c, "ragged": False, "counts": False}) if kind == "attend" else work(c)
        if full["bytes"] <= _MOST_BYTES[kind] and full["flops"] <= _MOST_FLOPS:
            # the plain form holds every logit and the whole cache in 32 bits
            if kind != "attend" or c["batch"] * c["max_len"] * max(c["heads"] * c["drafts"], c["kv_heads"] * dim) <= 1.2e9:
                return c


# ------------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, batch, heads, tokens, dim, dtype, token_major, scale=1.0):
    """N(0, scale^2) values [B, H, N, D], the memory behind them [B, N, H, D] if token_major."""
    shape = (batch, tokens, heads, dim) if token_major else (batch, heads, tokens, dim)
    x = torch.randn(shape, generator=g, device="cuda", dtype=F32).mul_(scale).to(dtype)
    return x.transpose(1, 2) if token_major else x


def _with_outliers(x, g):
    """A few channels of every head ten times as large, as keys have."""
    dim = x.shape[-1]
    at = torch.randint(0, dim, (max(1, dim // 32),), generator=g, device="cuda")
    gain = torch.ones(dim, device="cuda", dtype=F32)
    gain[at] = 10.0
    return (x.float() * gain).to(x.dtype)


def _pages_of(case, tokens):
    return -(-tokens // case["page"])


def _page_table(batch, pages, g):
    """Pages of the sequences, in no order."""
    return torch.randperm(batch * pages, generator=g, device="cuda").reshape(batch, pages).to(torch.int32)


def _slots(table, tokens, page):
    at = torch.arange(tokens, device="cuda")
    return (table.long()[:, at // page] * page + at % page).to(torch.int32)


def _empty_cache(case, pages):
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    kind = {"bf16": BF16, "e4m3": torch.uint8, "int8": torch.int8}[case["fmt"]]
    cache = {n: torch.zeros(shape, dtype=kind, device="cuda") for n in ("k", "v")}
    for n in ("k_scale", "v_scale"):
        cache[n] = None if case["fmt"] == "bf16" else torch.zeros(shape[:3], dtype=F32, device="cuda")
    return cache


def _filled_cache(case, pages, g):
    """A cache whose every slot holds a token: codes and scales of N(0, 1) rows."""
    cache = _empty_cache(case, pages)
    shape = tuple(cache["k"].shape)
    for n in ("k", "v"):
        x = torch.randn(shape, generator=g, device="cuda", dtype=BF16)
        if case["fmt"] == "bf16":
            cache[n] = x
            continue
        top = 1.0 + 3.0 * torch.rand(shape[:3], generator=g, device="cuda", dtype=F32)   # a row's largest magnitude
        if case["fmt"] == "e4m3":
            cache[n] = x.mul_(96.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
            cache[n + "_scale"] = torch.exp2(torch.floor(torch.log2(top)) - 8.0)
        else:
            cache[n] = x.mul_(40.0).clamp_(-127.0, 127.0).round_().to(torch.int8)
            cache[n + "_scale"] = top / 127.0
    return cache


def _trees(case, seed):
    """uint8 [B, T, T]: a drafted token sees itself and its ancestors in a random tree; and the
    drafted tokens that each sequence has."""
    r = np.random.RandomState(seed % (1 << 31))
    batch, t = case["batch"], case["drafts"]
    mask = np.zeros((batch, t, t), dtype=np.uint8)
    parent = np.array([[0] + [r.randint(max(0, n - 6), n) for n in range(1, t)] for _ in range(batch)])
    for n in range(t):
        if n:
            mask[:, n] = mask[np.arange(batch), parent[:, n]]
        mask[:, n, n] = 1
    counts = r.randint(1, t + 1, size=batch) if case["counts"] else np.full(batch, t)
    return mask, counts.astype(np.int32)


def _lengths(case, seed):
    """Cached tokens of each sequence; the first one is the longest."""
    r = np.random.RandomState(seed % (1 << 31))
    top, batch = case["max_len"], case["batch"]
    n = np.full(batch, top, dtype=np.int64)
    if case["ragged"]:
        n[1:] = np.exp(r.uniform(math.log(max(1.0, top / 64.0)), math.log(top + 1.0), size=batch - 1)).astype(np.int64)
    return np.minimum(n, top).astype(np.int32)


def prepare(case, seed):
    g = _generator(seed)
    b, t, dim = case["batch"], case.get("tokens", case.get("drafts")), case["dim"]
    st = {"case": case}
    if case["kind"] == "rotary":
        kind = _TYPES[case["dtype"]]
        st["q"] = _normal(g, b, case["heads"], t, dim, kind, case["token_major"])
        st["k"] = _normal(g, b, case["kv_heads"], t, dim, kind, case["token_major"])
        first = torch.randint(0, case["start"] + 1, (b, 1), generator=g, device="cuda")
        st["positions"] = (first + torch.arange(t, device="cuda")).to(torch.int32)
        st["freq"], st["magnitude"] = _frequencies(case)
        if own:
            import paper_2606_23743_amd as sva
            st["plan"] = sva.rotary_plan(head_dim=dim, rot_dim=case["rot"], layout=case["layout"], base=case["base"],
                                         scaling=case["scaling"], factor=case["factor"], original_len=case["orig"])
    elif case["kind"] == "write":
        kind = _TYPES[case["dtype"]]
        st["k"] = _with_outliers(_normal(g, b, case["kv_heads"], t, dim, kind, case["token_major"]), g)
        st["v"] = _normal(g, b, case["kv_heads"], t, dim, kind, case["token_major"])
        table = _page_table(b, _pages_of(case, t), g)
        st["slots"] = _slots(table, t, case["page"])
        st["cache"] = _empty_cache(case, table.numel())
    elif case["kind"] == "read":
        table = _page_table(b, _pages_of(case, t), g)
        st["slots"] = _slots(table, t, case["page"])
        st["cache"] = _filled_cache(case, table.numel(), g)
    else:
        st["table"] = _page_table(b, _pages_of(case, case["max_len"]), g)
        st["cache"] = _filled_cache(case, st["table"].numel(), g)
        st["lengths"] = torch.from_numpy(_lengths(case, seed)).cuda()
        st["q"] = _normal(g, b, case["heads"], t, dim, BF16, case["token_major"], 1.5)
        st["k_new"] = _normal(g, b, case["kv_heads"], t, dim, BF16, case["token_major"])
        st["v_new"] = _normal(g, b, case["kv_heads"], t, dim, BF16, case["token_major"])
        mask, counts = _trees(case, seed)
        st["mask"], st["counts"] = torch.from_numpy(mask).cuda(), torch.from_numpy(counts).cuda()
        # what a program keeps: rows behind a sequence's drafts stay as they are here
        st["out"] = torch.zeros_like(st["q"], dtype=_TYPES[case["out"]])
        st["lse"] = torch.zeros((b, case["heads"], t), dtype=F32, device="cuda") if case["lse"] else None
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    if not own:
        return {"rotary": _rotary_plain, "write": _write_plain, "read": _read_plain, "attend": _attend_plain}[case["kind"]](st)
    import paper_2606_23743_amd as sva
    if case["kind"] == "rotary":
        return sva.rotary(st["plan"], st["positions"], st["q"], st["k"], backward=case["backward"])
    if case["kind"] == "write":
        sva.cache_write(st["cache"], st["k"], st["v"], st["slots"])
        return _cache_outputs(case, st["cache"])
    if case["kind"] == "read":
        return sva.cache_read(st["cache"], st["slots"], dtype=case["dtype"])
    out, lse = sva.cache_attention(st["cache"], st["q"], st["table"], st["lengths"], st["k_new"], st["v_new"],
                                   mask=st["mask"], counts=st["counts"] if case["counts"] else None,
                                   out=st["out"], lse=st["lse"])
    return (out, lse) if case["lse"] else out


def _cache_outputs(case, cache):
    """The cache's own buffers; e4m3 codes as the values they are."""
    if case["fmt"] == "bf16":
        return cache["k"], cache["v"]
    k, v = cache["k"], cache["v"]
    if case["fmt"] == "e4m3":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    return k, cache["k_scale"], v, cache["v_scale"]


def _frequencies(case):
    """Radians per position of each pair (float64 [rot / 2]) and the factor on cosine and sine."""
    rot, base, s = case["rot"], case["base"], case["factor"]
    at = torch.arange(rot // 2, dtype=F64, device="cuda")
    if case["scaling"] == "ntk" and rot > 2:
        base = base * s ** (rot / (rot - 2.0))
    f = base ** (-2.0 * at / rot)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "yarn":
        turns = case["orig"] * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / s * (1.0 - keep), 0.1 * math.log(s) + 1.0
    return f, 1.0


def _rotary_plain(st):
    case, rot = st["case"], st["case"]["rot"]
    angle = st["positions"].to(F64)[:, None, :, None] * st["freq"]       # far positions need 64 bits
    cos, sin = (angle.cos() * st["magnitude"]).float(), (angle.sin() * st["magnitude"]).float()
    sin = -sin if case["backward"] else sin

    def turn(x):
        y = x.float()
        if case["layout"] == "half":
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            t = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            t = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
        return torch.cat((t, y[..., rot:]), dim=-1).to(x.dtype)

    return turn(st["q"]), turn(st["k"])


def _write_plain(st):
    case, cache = st["case"], st["cache"]
    slots = st["slots"].long().flatten()
    page, off = slots // case["page"], slots % case["page"]
    for n in ("k", "v"):
        x = st[n].transpose(1, 2).flatten(0, 1).float()                   # [tokens, heads, dim]
        if case["fmt"] == "bf16":
            cache[n][page, :, off] = x.to(BF16)
            continue
        top = x.abs().amax(dim=-1)
        if case["fmt"] == "e4m3":
            part, e = torch.frexp(top)                                    # top = part * 2^e, part in [0.5, 1)
            e = torch.where(top > 0, torch.where(part <= 0.875, e - 9, e - 8), 0)
            scale = torch.exp2(e.float())
            cache[n].view(torch.float8_e4m3fn)[page, :, off] = (x / scale[..., None]).to(torch.float8_e4m3fn)
        else:
            # in 64 bits: a quotient next to a half step has to fall on its own side
            scale = torch.where(top > 0, top.double() / 127.0, 1.0).float()
            cache[n][page, :, off] = (x.double() / scale.double()[..., None]).round().to(torch.int8)
        cache[n + "_scale"][page, :, off] = scale
    return _cache_outputs(case, cache)


def _values(case, cache, n):
    x = cache[n]
    x = (x.view(torch.float8_e4m3fn) if case["fmt"] == "e4m3" else x).float()
    return x if case["fmt"] == "bf16" else x * cache[n + "_scale"][..., None]


def _read_plain(st):
    case = st["case"]
    slots = st["slots"].long()
    page, off = slots // case["page"], slots % case["page"]

    def back(n):
        rows = {m: None if st["cache"][m] is None else st["cache"][m][page, :, off] for m in (n, n + "_scale")}
        return _values(case, rows, n).transpose(1, 2).to(_TYPES[case["dtype"]]).contiguous()

    return back("k"), back("v")


def _attend_plain(st):
    case, cache = st["case"], st["cache"]
    b, h, kv, t, dim = case["batch"], case["heads"], case["kv_heads"], case["drafts"], case["dim"]
    table = st["table"].long()

    def cached(n):
        rows = {m: None if cache[m] is None else cache[m][table] for m in (n, n + "_scale")}
        return _values(case, rows, n).permute(0, 2, 1, 3, 4).reshape(b, kv, -1, dim)

    k, v = cached("k"), cached("v")
    q = st["q"].float().reshape(b, kv, h // kv * t, dim) / math.sqrt(dim)
    seen = (torch.arange(k.shape[2], device="cuda") < st["lengths"][:, None])[:, None, None, :]
    s = torch.where(seen, q @ k.transpose(2, 3), -math.inf)
    mask = (st["mask"] != 0)[:, None, None].expand(b, kv, h // kv, t, t).reshape(b, kv, -1, t)
    s_new = torch.where(mask, q @ st["k_new"].float().transpose(2, 3), -math.inf)
    top = torch.maximum(s.amax(dim=-1, keepdim=True), s_new.amax(dim=-1, keepdim=True))
    w, w_new = torch.exp(s - top), torch.exp(s_new - top)
    total = w.sum(dim=-1, keepdim=True) + w_new.sum(dim=-1, keepdim=True)
    o = (w @ v + w_new @ st["v_new"].float()) / total
    here = (torch.arange(t, device="cuda") < st["counts"][:, None])[:, None, :, None]
    out = torch.where(here, o.reshape(b, h, t, dim), 0.0).to(st["out"].dtype)
    lse = torch.where(here, (top + total.log()).reshape(b, h, t, 1), 0.0)[..., 0]
    return (out, lse) if case["lse"] else out


# ------------------------------------------------------- work and definitions

def work(case):
    b, dim = case["batch"], case["dim"]
    if case["kind"] == "rotary":
        item = 2 if case["dtype"] == "bf16" else 4
        heads, n = case["heads"] + case["kv_heads"], b * case["tokens"]
        return {"bytes": 2 * n * heads * dim * item + 4 * n, "flops": 3 * n * heads * case["rot"]}
    row = {"bf16": 2 * dim, "e4m3": dim + 4, "int8": dim + 4}[case["fmt"]]
    if case["kind"] in ("write", "read"):
        n = b * case["tokens"]
        item = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * case["kv_heads"] * (dim * item + row) + 4 * n, "flops": 2 * n * case["kv_heads"] * dim}
    # lengths are drawn with the inputs: their mean over seeds where they are ragged
    top = case["max_len"]
    low = max(1.0, top / 64.0)
    mean = (top + 1.0 - low) / math.log((top + 1.0) / low) if case["ragged"] else top
    keys = top + (b - 1) * mean
    t = (case["drafts"] + 1) / 2 if case["counts"] else case["drafts"]
    out = 2 if case["out"] == "bf16" else 4
    return {"bytes": keys * case["kv_heads"] * 2 * row + b * t * dim * (case["heads"] * (2 + out) + case["kv_heads"] * 4),
            "flops": 4 * case["heads"] * dim * t * (keys + b * t)}


def exact(case, seed):
    st = prepare(case, seed)
    return {"rotary": _rotary_exact, "write": _write_exact, "read": _read_exact, "attend": _attend_exact}[case["kind"]](st)


def _rotary_exact(st):
    """Pair i of a row at position p, as a complex number, times m exp(+-i p f_i)."""
    case, rot, s = st["case"], st["case"]["rot"], st["case"]["factor"]
    i = np.arange(rot // 2, dtype=np.float64)
    base = case["base"] * (s ** (rot / (rot - 2.0)) if case["scaling"] == "ntk" and rot > 2 else 1.0)
    f, m = np.power(base, -2.0 * i / rot), 1.0
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "yarn":
        keep = np.clip((case["orig"] * f / (2.0 * np.pi) - 1.0) / 31.0, 0.0, 1.0)
        f, m = f / s * (1.0 - keep) + f * keep, 0.1 * math.log(s) + 1.0
    angle = st["positions"].double().unsqueeze(-1) * torch.from_numpy(f).cuda()
    z = torch.polar(torch.full_like(angle, m), -angle if case["backward"] else angle).unsqueeze(1)

    def turn(x):
        y = x.double().clone()
        first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        w = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * z
        y[..., first], y[..., second] = w.real, w.imag
        return y

    return turn(st["q"]), turn(st["k"])


def _write_exact(st):
    case, cache = st["case"], st["cache"]
    place = st["slots"].long()
    outs = []
    for n in ("k", "v"):
        x = st[n].double()
        pages, kv, page, dim = cache[n].shape
        codes = torch.zeros((pages * page, kv, dim), dtype=F64, device="cuda")
        scales = torch.zeros((pages * page, kv), dtype=F64, device="cuda")
        top = x.abs().max(dim=-1).values
        if case["fmt"] == "bf16":
            codes[place] = x.permute(0, 2, 1, 3)
            outs.append(codes.reshape(pages, page, kv, dim).transpose(1, 2))
            continue
        if case["fmt"] == "e4m3":
            e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))     # then to the right side of a power of two
            e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)
            e = torch.where(448.0 * torch.exp2(e) < top, e + 1, e)
            scale = torch.where(top > 0, torch.exp2(e), 1.0)
            y = x / scale[..., None]
            step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=1e-300))), min=-6.0) - 3.0)
            y = torch.round(y / step) * step
        else:
            scale = torch.where(top > 0, top / 127.0, 1.0).float().double()   # a scale is a float32 by definition
            y = torch.round(x / scale[..., None])
        codes[place] = y.permute(0, 2, 1, 3)
        scales[place] = scale.permute(0, 2, 1)
        codes = codes.reshape(pages, page, kv, dim).transpose(1, 2)
        outs += [codes if case["fmt"] == "e4m3" else codes.to(torch.int8), scales.reshape(pages, page, kv).transpose(1, 2)]
    return tuple(outs)


def _code_values(case, codes):
    """float64 values of codes: an e4m3 byte is sign, four exponent bits (bias 7), three of the fraction."""
    if case["fmt"] != "e4m3":
        return codes.double()
    c = codes.long()
    e, frac = (c >> 3) & 15, (c & 7).double() / 8.0
    size = torch.where(e > 0, (1.0 + frac) * torch.exp2(e.double() - 7.0), frac * 2.0 ** -6)
    return torch.where(c >= 128, -size, size)


def _tokens_exact(case, cache, n, slots):
    """float64 [tokens, kv_heads, dim] of the tokens at these slots."""
    rows = cache[n].transpose(1, 2).flatten(0, 1)[slots]
    x = _code_values(case, rows)
    return x if cache[n + "_scale"] is None else x * cache[n + "_scale"].transpose(1, 2).flatten(0, 1)[slots].double().unsqueeze(-1)


def _read_exact(st):
    case = st["case"]
    slots = st["slots"].long()
    return tuple(_tokens_exact(case, st["cache"], n, slots.flatten()).reshape(*slots.shape, case["kv_heads"], case["dim"])
                 .transpose(1, 2) for n in ("k", "v"))


def _attend_exact(st):
    """Sequence by sequence: softmax over the visible keys alone."""
    case, cache = st["case"], st["cache"]
    b, h, kv, t, dim = case["batch"], case["heads"], case["kv_heads"], case["drafts"], case["dim"]
    out = torch.zeros((b, h, t, dim), dtype=F64, device="cuda")
    lse = torch.zeros((b, h, t), dtype=F64, device="cuda")
    lengths, counts = st["lengths"].tolist(), st["counts"].tolist()
    for i in range(b):
        n, c = lengths[i], counts[i] if case["counts"] else t
        slots = _slots(st["table"][i:i + 1], n, case["page"])[0].long()
        hidden = torch.zeros((c, n + c), dtype=torch.bool, device="cuda")
        hidden[:, n:] = st["mask"][i, :c, :c] == 0
        for j in range(kv):
            one = {m: None if cache[m] is None else cache[m][:, j:j + 1] for m in cache}
            k = torch.cat((_tokens_exact(case, one, "k", slots)[:, 0], st["k_new"][i, j, :c].double()))
            v = torch.cat((_tokens_exact(case, one, "v", slots)[:, 0], st["v_new"][i, j, :c].double()))
            heads = slice(j * (h // kv), (j + 1) * (h // kv))
            s = torch.matmul(st["q"][i, heads, :c].double().reshape(-1, dim), k.t()).reshape(-1, c, n + c) * dim ** -0.5
            s = s.masked_fill(hidden, -math.inf)
            out[i, heads, :c] = torch.matmul(torch.softmax(s, dim=-1).reshape(-1, n + c), v).reshape(-1, c, dim)
            lse[i, heads, :c] = torch.logsumexp(s, dim=-1)
    return (out, lse) if case["lse"] else out
