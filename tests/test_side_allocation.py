"""Which stream the memory belongs to that a call of the binding allocates, on the CPU.

The caching allocator hands out a block that was freed on a stream while that stream's
kernels may still use it: safe for what is launched on that stream afterwards, and for
nothing else.  So a call that is given a stream has to allocate its workspace and its
outputs on that stream, and to mark the outputs, which the caller goes on to use, for
the current one.  Here torch and the library are stand-ins that note the stream of every
allocation and marking; the calls are the binding's own."""
import contextlib
from types import SimpleNamespace

import pytest
import torch as real

from paper_2606_23743_amd import _lib

pytestmark = pytest.mark.cpu

SIZES = {real.bfloat16: 2, real.float32: 4, real.float64: 8, real.int32: 4, real.uint8: 1, real.int8: 1, real.bool: 1}


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Tensor:
    """A contiguous device tensor without memory."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype, stream=None):
        self.shape, self.dtype, self.made_on, self.marks = real.Size(shape), dtype, stream, set()

    def dim(self):
        return len(self.shape)

    def stride(self, d=None):
        s, out = 1, []
        for n in reversed(self.shape):
            out.insert(0, s)
            s *= n
        return tuple(out) if d is None else out[d]

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return SIZES[self.dtype]

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, s):
        self.marks.add(s.cuda_stream)


class World:
    """The stand-ins: a current stream (100), a side stream (200), every tensor made."""

    def __init__(self):
        self.current, self.side, self.made = [Stream(100)], Stream(200), []

        def empty(*shape, dtype, device=None):
            shape = shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape
            t = Tensor(shape, dtype, self.current[-1].cuda_stream)
            self.made.append(t)
            return t

        @contextlib.contextmanager
        def stream(s):
            self.current.append(s)
            yield
            self.current.pop()

        cuda = SimpleNamespace(current_device=lambda: 0, is_initialized=lambda: True, Stream=Stream, stream=stream,
                               current_stream=lambda *a: self.current[-1], ExternalStream=Stream)
        c = SimpleNamespace(_cuda_getDevice=lambda: 0,
                            _cuda_getCurrentRawStream=lambda dev: self.current[-1].cuda_stream)
        names = ("bfloat16", "float32", "float64", "int32", "uint8", "int8", "bool")
        self.torch = SimpleNamespace(Tensor=Tensor, cuda=cuda, _C=c, empty=lambda shape, **kw: empty(shape, **kw),
                                     empty_like=lambda t, dtype=None: empty(t.shape, dtype=dtype or t.dtype),
                                     **{n: getattr(real, n) for n in names})
        real_lib = _lib.load()

        def entry(name):
            host = getattr(real_lib, name)
            if any(part in name for part in ("workspace", "num_blocks", "max_keep", "keep_count", "padded", "code_dim")):
                return host                              # host only: the library's own
            return lambda *a: 0

        self.lib = type("Lib", (), {"__getattr__": lambda s, name: entry(name)})()

    def t(self, *shape, dtype=real.bfloat16):
        return Tensor(shape, dtype)


@pytest.fixture
def world(monkeypatch):
    w = World()
    monkeypatch.setattr(_lib, "_torch_module", w.torch)
    monkeypatch.setattr(_lib, "load", lambda *a: w.lib)
    monkeypatch.setattr(_lib, "_workspace_bytes", {})
    return w


def calls(w):
    """name, call(**kw) that leaves everything to be allocated, and how many outputs it returns."""
    i32, f32, u8, f64 = real.int32, real.float32, real.uint8, real.float64
    prob = _lib.problem(1, 2, 4096, 64, (1, 64, 64), 64)
    sel = _lib.select_topk(topk=4)
    q = w.t(1, 2, 4096, 64)
    pool, idx, cnt = w.t(1, 2, 64, 64, dtype=f32), w.t(1, 2, 64, 4, dtype=i32), w.t(1, 2, 64, dtype=i32)
    npad, dp = _lib.fp8_padded_len(prob), _lib.fp8_code_dim(prob)
    quant = {"q8": w.t(1, 2, npad, dp, dtype=u8), "k8": w.t(1, 2, npad, dp, dtype=u8),
             "v8": w.t(1, 2, npad // 64, dp, 64, dtype=u8), "q_exp": w.t(1, 2, 64, dtype=i32),
             "k_exp": w.t(1, 2, 64, dtype=i32), "v_exp": w.t(1, 2, dp, dtype=i32), "k_mean": w.t(1, 2, 64)}
    x = w.t(1, 300, 256)
    keep = _lib.token_keep_count(_lib.tokens(1, 300, 256), 0.5)
    plan = {"head_dim": 64, "rot_dim": 64, "layout": "half", "magnitude": 1.0, "freq": w.t(32, dtype=f64)}
    cache = {"k": w.t(64, 2, 64, 64, dtype=u8), "v": w.t(64, 2, 64, 64, dtype=u8),
             "k_scale": w.t(64, 2, 64, dtype=f32), "v_scale": w.t(64, 2, 64, dtype=f32)}
    return [
        ("pool_blocks", lambda **kw: _lib.pool_blocks(prob, q, q, **kw), 2),
        ("qknorm_rope_pool", lambda **kw: _lib.qknorm_rope_pool(prob, q, q, w.t(64, dtype=f32), w.t(64, dtype=f32), **kw), 4),
        ("select_blocks", lambda **kw: _lib.select_blocks(prob, sel, pool, pool, want_mask=True, **kw), 3),
        ("sparse_attention", lambda **kw: _lib.sparse_attention(prob, q, q, q, idx, cnt, want_lse=True, **kw), 2),
        ("dense_attention", lambda **kw: _lib.dense_attention(prob, q, q, q, want_lse=True, **kw), 2),
        ("block_moments", lambda **kw: _lib.block_moments(prob, q, q, **kw), 3),
        ("sparse_attention_remainder",
         lambda **kw: _lib.sparse_attention_remainder(prob, q, q, q, pool, pool, idx, cnt, want_lse=True, **kw), 2),
        ("quantize_fp8", lambda **kw: tuple(_lib.quantize_fp8(prob, q, q, q, **kw).values()), 7),
        ("sparse_attention_fp8", lambda **kw: _lib.sparse_attention_fp8(prob, quant, idx, cnt, want_lse=True, **kw), 2),
        ("dense_attention_fp8", lambda **kw: _lib.dense_attention_fp8(prob, quant, want_lse=True, **kw), 2),
        ("token_select", lambda **kw: _lib.token_select(x, 0.5, **kw), 3),
        ("token_select_noalloc", lambda **kw: _lib.token_select_noalloc(x, 0.5, **kw), 3),
        ("token_gather", lambda **kw: (_lib.token_gather(x, w.t(1, keep, dtype=i32), **kw),), 1),
        ("token_scatter", lambda **kw: (_lib.token_scatter(w.t(1, keep, 256), w.t(1, 300, dtype=i32), x, **kw),), 1),
        ("rotary", lambda **kw: _lib.rotary(plan, w.t(1, 9, dtype=i32), w.t(1, 4, 9, 64), w.t(1, 2, 9, 64), **kw), 2),
        ("cache_read", lambda **kw: _lib.cache_read(cache, w.t(1, 9, dtype=i32), **kw), 2),
        ("cache_attention",
         lambda **kw: _lib.cache_attention(cache, w.t(1, 4, 3, 64), w.t(1, 64, dtype=i32), w.t(1, dtype=i32),
                                           w.t(1, 2, 3, 64), w.t(1, 2, 3, 64), want_lse=True, **kw), 2),
    ]


NAMES = ["pool_blocks", "qknorm_rope_pool", "select_blocks", "sparse_attention", "dense_attention", "block_moments",
         "sparse_attention_remainder", "quantize_fp8", "sparse_attention_fp8", "dense_attention_fp8", "token_select",
         "token_select_noalloc", "token_gather", "token_scatter", "rotary", "cache_read", "cache_attention"]
WORKSPACE = {"sparse_attention_remainder", "token_select", "cache_attention"}


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("handle", [False, True])
def test_memory_belongs_to_the_stream_that_uses_it_first(world, name, handle):
    assert [n for n, _, _ in calls(world)] == NAMES
    call, outputs = next((f, n) for m, f, n in calls(world) if m == name)
    world.made.clear()
    got = call(stream=world.side.cuda_stream if handle else world.side)
    assert len(got) == outputs and len(world.made) == outputs + (name in WORKSPACE)
    assert len(world.current) == 1                           # the current stream is as it was
    for t in world.made:
        assert t.made_on == 200, "allocated on another stream than the call's"
    for t in got:
        assert 100 in t.marks, "the caller's use of an output is not marked"


@pytest.mark.parametrize("name", NAMES)
def test_without_a_side_stream_nothing_changes(world, name):
    call = next(f for m, f, _ in calls(world) if m == name)
    for kw in ({}, {"stream": world.current[0]}):
        world.made.clear()
        call(**kw)
        assert world.made and all(t.made_on == 100 and not t.marks for t in world.made)


def test_the_stand_in_covers_every_call_with_a_stream():
    import inspect
    takes = {n for n, f in inspect.getmembers(_lib, inspect.isfunction)
             if not n.startswith("_") and "stream" in inspect.signature(f).parameters}
    assert takes - set(NAMES) == {"cache_write"}             # allocates nothing
