"""ctypes binding of libsva.so (include/sva.h).  Argument marshalling only:
every step of the path runs in the library's HIP kernels.  torch supplies device
memory and the current stream; nothing here computes on the host, and there is
no fallback -- a missing or unloadable library raises.

A call with stream= (a torch stream or a handle) is launched there.  The caller
puts that stream behind the work that makes the inputs, and the work that uses the
outputs behind that stream; memory that the call allocates needs no such order.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsva.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "sva.h")

SVA_OK, SVA_ERR_INVALID_ARG, SVA_ERR_SHAPE, SVA_ERR_ALIGNMENT, SVA_ERR_UNSUPPORTED, SVA_ERR_HIP = range(6)
SVA_BF16, SVA_F32 = 0, 1
SVA_SELECT_TOPK, SVA_SELECT_CUMMASS = 0, 1
SVA_SELECT_MAX_BLOCKS = 2048
SVA_ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
SVA_ROTARY_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
SVA_CACHE_FORMATS = {"bf16": 0, "e4m3": 1, "int8": 2}
SVA_CACHE_MAX_QUERIES = 1024


class SvaError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


class Problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("grid_t", ctypes.c_int32), ("grid_h", ctypes.c_int32),
                ("grid_w", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("softmax_scale", ctypes.c_double), ("out_dtype", ctypes.c_int32)]


class RopeParams(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_double), ("rope_base", ctypes.c_double)]


class Tokens(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("channels", ctypes.c_int32)]


class Fp8Tensors(ctypes.Structure):
    _fields_ = [("q8", ctypes.c_void_p), ("k8", ctypes.c_void_p), ("v8", ctypes.c_void_p),
                ("q_exp", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("k_mean", ctypes.c_void_p)]


class SelectParams(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("keep_ratio", ctypes.c_double), ("topk", ctypes.c_int32),
                ("mass_threshold", ctypes.c_double), ("max_keep_ratio", ctypes.c_double),
                ("force_first_frame", ctypes.c_int32)]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("heads", ctypes.c_int32), ("stride_b", ctypes.c_int64),
                ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


class RotarySpec(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("original_len", ctypes.c_double), ("beta_fast", ctypes.c_double),
                ("beta_slow", ctypes.c_double), ("magnitude", ctypes.c_double)]


class RotaryParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("backward", ctypes.c_int32), ("magnitude", ctypes.c_double)]


class Cache(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class CacheQuery(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("queries", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("softmax_scale", ctypes.c_double), ("out_dtype", ctypes.c_int32)]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libsva.so once; raise if it is missing (build it with
    `python -m paper_2606_23743_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build the HIP library first "
                           "(python -m paper_2606_23743_amd.build)")
    lib = ctypes.CDLL(path)
    P, S = ctypes.POINTER(Problem), ctypes.POINTER(SelectParams)
    vp, i32p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)
    i32, i64, HP, CP = ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(Heads), ctypes.POINTER(Cache)
    sig = {
        "sva_num_blocks": [P, i32p],
        "sva_max_keep": [P, S, i32p],
        "sva_pool_blocks": [P, vp, vp, vp, vp, vp],
        "sva_qknorm_rope_pool": [P, ctypes.POINTER(RopeParams), vp, vp, vp, vp, vp, vp, vp, vp, vp],
        "sva_select_blocks": [P, S, vp, vp, ctypes.c_int32, vp, vp, vp, vp],
        "sva_sparse_attention": [P, vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp],
        "sva_dense_attention": [P, vp, vp, vp, vp, vp, vp],
        "sva_remainder_workspace": [P, ctypes.POINTER(ctypes.c_size_t)],
        "sva_remainder_workspace_heads": [P, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)],
        "sva_block_moments": [P, vp, vp, vp, vp, vp, vp],
        "sva_sparse_attention_remainder": [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int32, vp,
                                           ctypes.c_size_t, vp, vp, vp],
        "sva_token_keep_count": [ctypes.POINTER(Tokens), ctypes.c_double, i32p],
        "sva_token_select_workspace": [ctypes.POINTER(Tokens), ctypes.POINTER(ctypes.c_size_t)],
        "sva_token_select": [ctypes.POINTER(Tokens), ctypes.c_double, vp, vp, vp, vp, vp,
                             ctypes.c_size_t, vp],
        "sva_token_select_noalloc": [ctypes.POINTER(Tokens), ctypes.c_double, vp, vp, vp, vp, vp],
        "sva_token_gather": [ctypes.POINTER(Tokens), ctypes.c_int32, vp, vp, vp, vp],
        "sva_token_scatter": [ctypes.POINTER(Tokens), ctypes.c_int32, vp, vp, vp, vp, vp],
        "sva_fp8_padded_len": [P, i32p],
        "sva_fp8_code_dim": [P, i32p],
        "sva_quantize_fp8": [P, vp, vp, vp, ctypes.POINTER(Fp8Tensors), vp],
        "sva_sparse_attention_fp8": [P, ctypes.POINTER(Fp8Tensors), vp, vp, ctypes.c_int32, vp, vp, vp],
        "sva_dense_attention_fp8": [P, ctypes.POINTER(Fp8Tensors), vp, vp, vp],
        "sva_rotary_frequencies": [ctypes.POINTER(RotarySpec), ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_double)],
        "sva_rotary": [ctypes.POINTER(RotaryParams), vp, vp, i64, HP, HP, HP, HP, vp],
        "sva_cache_write": [CP, i32, i32, i32, HP, HP, vp, i64, vp],
        "sva_cache_read": [CP, i32, i32, i32, vp, i64, HP, HP, vp],
        "sva_cache_attention_workspace": [CP, ctypes.POINTER(CacheQuery), ctypes.POINTER(ctypes.c_size_t)],
        "sva_cache_attention": [CP, ctypes.POINTER(CacheQuery), HP, vp, vp, HP, HP, vp, i64, vp, vp,
                                ctypes.c_size_t, HP, vp, vp],
        "sva_status_string": [ctypes.c_int],
        "sva_version": [],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_char_p if name == "sva_status_string" else ctypes.c_int
    _lib = lib
    return lib


def header_functions(header: str = HEADER):
    """Names of the functions include/sva.h declares."""
    text = open(header).read()
    return sorted(set(re.findall(r"^\s*(?:const\s+char\*|int)\s+(sva_\w+)\s*\(", text, re.M)))


def status_string(status: int) -> str:
    try:
        return load().sva_status_string(int(status)).decode()
    except Exception:  # pragma: no cover - only while reporting another error
        return "?"


def _check(status: int, what: str):
    if status != SVA_OK:
        raise SvaError(status, what)


# ----------------------------------------------------------------- parameters

def problem(batch, heads, seq_len, head_dim, grid, block_size, softmax_scale=0.0,
            out_dtype="bf16") -> Problem:
    t, h, w = grid
    return Problem(batch, heads, seq_len, head_dim, t, h, w, block_size, float(softmax_scale),
                   SVA_F32 if out_dtype in ("f32", "float32", SVA_F32) else SVA_BF16)


def problem_for(wl, out_dtype="bf16", softmax_scale=0.0) -> Problem:
    return problem(wl.batch, wl.heads, wl.seq_len, wl.head_dim, (wl.grid_t, wl.grid_h, wl.grid_w),
                   wl.block, softmax_scale, out_dtype)


def select_topk(keep_ratio: float = 0.0, topk: int = 0) -> SelectParams:
    return SelectParams(SVA_SELECT_TOPK, float(keep_ratio), int(topk), 0.0, 0.0, 0)


def select_mass(tau: float, max_keep_ratio: float, force_first_frame: bool) -> SelectParams:
    return SelectParams(SVA_SELECT_CUMMASS, 0.0, 0, float(tau), float(max_keep_ratio),
                        1 if force_first_frame else 0)


def select_for(wl, keep_ratio: Optional[float] = None) -> SelectParams:
    if wl.mode == "mass":
        return select_mass(wl.mass_threshold, wl.max_keep_ratio, wl.force_first_frame)
    if keep_ratio is not None:
        return select_topk(keep_ratio, 0)
    return select_topk(wl.keep_ratio, wl.topk)


def num_blocks(prob: Problem) -> int:
    out = ctypes.c_int32()
    _check(load().sva_num_blocks(ctypes.byref(prob), ctypes.byref(out)), "sva_num_blocks")
    return out.value


def max_keep(prob: Problem, sel: SelectParams) -> int:
    out = ctypes.c_int32()
    _check(load().sva_max_keep(ctypes.byref(prob), ctypes.byref(sel), ctypes.byref(out)), "sva_max_keep")
    return out.value


# ------------------------------------------------------------- device calls

# A small call's time is this module's own: three launches of 3 to 9 us went out
# every 41 us.  So torch is looked up once, a tensor that is as it should be
# passes one test, tensors made here are not tested again, and the current stream
# is asked for as a handle, without a stream object around it.
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        torch = _torch()
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _side_stream(stream):
    """The stream a call was given, as a torch stream object, when it is not
    the current stream (None otherwise)."""
    torch = _torch()
    if stream is None:
        return None
    cur = torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return None if stream.cuda_stream == cur else stream
    h = int(stream.cuda_stream if hasattr(stream, "cuda_stream") else stream)
    return None if h == cur else torch.cuda.ExternalStream(h)


def _output(stream, make, *args, **kw):
    """make(*args, **kw), an output that a call on `stream` writes.  The caching
    allocator hands out memory that was freed on a stream while kernels of that
    stream may still use it, which is in order for that stream alone: so the memory
    is taken on the call's stream, and marked for the current one, where the
    caller uses (and frees) it."""
    s = None if stream is None else _side_stream(stream)
    if s is None:
        return make(*args, **kw)
    torch = _torch()
    with torch.cuda.stream(s):
        x = make(*args, **kw)
    x.record_stream(torch.cuda.current_stream())
    return x


def _scratch(stream, nbytes, device):
    """A workspace, which no other stream uses: taken on the call's stream."""
    torch = _torch()
    s = _side_stream(stream)
    if s is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(s):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _record(stream, *tensors):
    """Mark every tensor a call reads or writes as in use on the call's stream
    when that is not the current stream: the caching allocator then keeps the
    memory of a tensor freed meanwhile (an input or an output of the caller's,
    who drops it) from being handed to another allocation until the work
    enqueued on that stream has finished."""
    if stream is None:
        return
    s = _side_stream(stream)
    if s is None:
        return
    for x in tensors:
        if isinstance(x, dict):
            _record(stream, *x.values())
        elif x is not None:
            x.record_stream(s)


def _need(t, dtype, shape, name):
    torch = _torch()
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _qkv_shape(prob):
    return (prob.batch, prob.heads, prob.seq_len, prob.head_dim)


def pool_blocks(prob: Problem, q, k, q_pool=None, k_pool=None, stream=None) -> Tuple:
    torch = _torch()
    nb = num_blocks(prob)
    shp = _qkv_shape(prob)
    _need(q, torch.bfloat16, shp, "q")
    _need(k, torch.bfloat16, shp, "k")
    pshape = (prob.batch, prob.heads, nb, prob.head_dim)
    if q_pool is None:
        q_pool = _output(stream, torch.empty, pshape, dtype=torch.float32, device=q.device)
    else:
        _need(q_pool, torch.float32, pshape, "q_pool")
    if k_pool is None:
        k_pool = _output(stream, torch.empty, pshape, dtype=torch.float32, device=q.device)
    else:
        _need(k_pool, torch.float32, pshape, "k_pool")
    _check(load().sva_pool_blocks(ctypes.byref(prob), _ptr(q), _ptr(k), _ptr(q_pool), _ptr(k_pool),
                                  _stream(stream)), "sva_pool_blocks")
    _record(stream, q, k, q_pool, k_pool)
    return q_pool, k_pool


def qknorm_rope_pool(prob: Problem, q_in, k_in, gamma_q, gamma_k, eps: float = 1e-6,
                     rope_base: float = 10000.0, q_out=None, k_out=None, q_pool=None, k_pool=None,
                     stream=None) -> Tuple:
    """RMSNorm + 3-D RoPE of Q and K with the block summaries of the written
    values (sva_qknorm_rope_pool).  q_out / k_out may be q_in / k_in (in place)."""
    torch = _torch()
    nb = num_blocks(prob)
    shp = _qkv_shape(prob)
    _need(q_in, torch.bfloat16, shp, "q_in")
    _need(k_in, torch.bfloat16, shp, "k_in")
    _need(gamma_q, torch.float32, (prob.head_dim,), "gamma_q")
    _need(gamma_k, torch.float32, (prob.head_dim,), "gamma_k")
    if q_out is None:
        q_out = _output(stream, torch.empty_like, q_in)
    else:
        _need(q_out, torch.bfloat16, shp, "q_out")
    if k_out is None:
        k_out = _output(stream, torch.empty_like, k_in)
    else:
        _need(k_out, torch.bfloat16, shp, "k_out")
    pshape = (prob.batch, prob.heads, nb, prob.head_dim)
    if q_pool is None:
        q_pool = _output(stream, torch.empty, pshape, dtype=torch.float32, device=q_in.device)
    else:
        _need(q_pool, torch.float32, pshape, "q_pool")
    if k_pool is None:
        k_pool = _output(stream, torch.empty, pshape, dtype=torch.float32, device=q_in.device)
    else:
        _need(k_pool, torch.float32, pshape, "k_pool")
    rp = RopeParams(float(eps), float(rope_base))
    _check(load().sva_qknorm_rope_pool(ctypes.byref(prob), ctypes.byref(rp), _ptr(q_in), _ptr(k_in),
                                       _ptr(gamma_q), _ptr(gamma_k), _ptr(q_out), _ptr(k_out),
                                       _ptr(q_pool), _ptr(k_pool), _stream(stream)),
           "sva_qknorm_rope_pool")
    _record(stream, q_in, k_in, gamma_q, gamma_k, q_out, k_out, q_pool, k_pool)
    return q_out, k_out, q_pool, k_pool


def select_blocks(prob: Problem, sel: SelectParams, q_pool, k_pool, kmax: Optional[int] = None,
                  kv_idx=None, kv_count=None, want_mask: bool = False, mask=None, stream=None) -> Tuple:
    torch = _torch()
    nb = num_blocks(prob)
    pshape = (prob.batch, prob.heads, nb, prob.head_dim)
    _need(q_pool, torch.float32, pshape, "q_pool")
    _need(k_pool, torch.float32, pshape, "k_pool")
    if kmax is None:
        kmax = max_keep(prob, sel)
    dev = q_pool.device
    if kv_idx is None:
        kv_idx = _output(stream, torch.empty, (prob.batch, prob.heads, nb, kmax), dtype=torch.int32, device=dev)
    else:
        _need(kv_idx, torch.int32, (prob.batch, prob.heads, nb, kmax), "kv_idx")
    if kv_count is None:
        kv_count = _output(stream, torch.empty, (prob.batch, prob.heads, nb), dtype=torch.int32, device=dev)
    else:
        _need(kv_count, torch.int32, (prob.batch, prob.heads, nb), "kv_count")
    if want_mask and mask is None:
        mask = _output(stream, torch.empty, (prob.batch, prob.heads, nb, nb), dtype=torch.uint8, device=dev)
    if mask is not None:
        _need(mask, torch.uint8, (prob.batch, prob.heads, nb, nb), "mask")
    _check(load().sva_select_blocks(ctypes.byref(prob), ctypes.byref(sel), _ptr(q_pool), _ptr(k_pool),
                                    int(kmax), _ptr(kv_idx), _ptr(kv_count), _ptr(mask), _stream(stream)),
           "sva_select_blocks")
    _record(stream, q_pool, k_pool, kv_idx, kv_count, mask)
    return kv_idx, kv_count, mask


def _out_tensor(prob, like, out, stream):
    torch = _torch()
    dt = torch.float32 if prob.out_dtype == SVA_F32 else torch.bfloat16
    if out is None:
        return _output(stream, torch.empty, _qkv_shape(prob), dtype=dt, device=like.device)
    _need(out, dt, _qkv_shape(prob), "out")
    return out


def sparse_attention(prob: Problem, q, k, v, kv_idx, kv_count, out=None, want_lse: bool = False,
                     lse=None, stream=None) -> Tuple:
    torch = _torch()
    nb = num_blocks(prob)
    shp = _qkv_shape(prob)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, shp, n)
    kmax = kv_idx.shape[-1]
    _need(kv_idx, torch.int32, (prob.batch, prob.heads, nb, kmax), "kv_idx")
    _need(kv_count, torch.int32, (prob.batch, prob.heads, nb), "kv_count")
    out = _out_tensor(prob, q, out, stream)
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, shp[:3], dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, torch.float32, shp[:3], "lse")
    _check(load().sva_sparse_attention(ctypes.byref(prob), _ptr(q), _ptr(k), _ptr(v), _ptr(kv_idx),
                                       _ptr(kv_count), int(kmax), _ptr(out), _ptr(lse), _stream(stream)),
           "sva_sparse_attention")
    _record(stream, q, k, v, kv_idx, kv_count, out, lse)
    return out, lse


def remainder_workspace(prob: Problem, heads: Optional[int] = None) -> int:
    """Workspace bytes of sparse_attention_remainder: for all (batch, head)
    pairs in one pass (sva_remainder_workspace), or for passes of `heads`
    pairs (sva_remainder_workspace_heads)."""
    out = ctypes.c_size_t(0)
    if heads is None:
        _check(load().sva_remainder_workspace(ctypes.byref(prob), ctypes.byref(out)), "sva_remainder_workspace")
    else:
        _check(load().sva_remainder_workspace_heads(ctypes.byref(prob), int(heads), ctypes.byref(out)),
               "sva_remainder_workspace_heads")
    return out.value


def block_moments(prob: Problem, k, v, kbar=None, vbar=None, moments=None, stream=None) -> Tuple:
    """sva_block_moments: (kbar bf16 [B, H, nB, D], vbar bf16 [B, H, nB, D],
    moments bf16 [B, H, nB, D, D] with M[e][d] = sum_t V[t][e] (K[t][d] - kbar[d]))."""
    torch = _torch()
    nb = num_blocks(prob)
    shp = _qkv_shape(prob)
    B, H, _, D = shp
    for t, n in ((k, "k"), (v, "v")):
        _need(t, torch.bfloat16, shp, n)
    if kbar is None:
        kbar = _output(stream, torch.empty, (B, H, nb, D), dtype=torch.bfloat16, device=k.device)
    if vbar is None:
        vbar = _output(stream, torch.empty, (B, H, nb, D), dtype=torch.bfloat16, device=k.device)
    if moments is None:
        moments = _output(stream, torch.empty, (B, H, nb, D, D), dtype=torch.bfloat16, device=k.device)
    _need(kbar, torch.bfloat16, (B, H, nb, D), "kbar")
    _need(vbar, torch.bfloat16, (B, H, nb, D), "vbar")
    _need(moments, torch.bfloat16, (B, H, nb, D, D), "moments")
    _check(load().sva_block_moments(ctypes.byref(prob), _ptr(k), _ptr(v), _ptr(kbar), _ptr(vbar), _ptr(moments),
                                    _stream(stream)), "sva_block_moments")
    _record(stream, k, v, kbar, vbar, moments)
    return kbar, vbar, moments


def sparse_attention_remainder(prob: Problem, q, k, v, q_pool, k_pool, kv_idx, kv_count, out=None,
                               want_lse: bool = False, lse=None, workspace=None, stream=None) -> Tuple:
    """sva_sparse_attention_remainder: the kept blocks exactly plus the
    first-order remainder of the dropped ones.  workspace: a uint8 device
    tensor of remainder_workspace bytes (allocated when None), or of at least
    remainder_workspace(prob, 1), with which the (batch, head) pairs are done
    in groups of as many as fit."""
    torch = _torch()
    nb = num_blocks(prob)
    shp = _qkv_shape(prob)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, shp, n)
    _need(q_pool, torch.float32, (prob.batch, prob.heads, nb, prob.head_dim), "q_pool")
    _need(k_pool, torch.float32, (prob.batch, prob.heads, nb, prob.head_dim), "k_pool")
    kmax = kv_idx.shape[-1]
    _need(kv_idx, torch.int32, (prob.batch, prob.heads, nb, kmax), "kv_idx")
    _need(kv_count, torch.int32, (prob.batch, prob.heads, nb), "kv_count")
    out = _out_tensor(prob, q, out, stream)
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, shp[:3], dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, torch.float32, shp[:3], "lse")
    if workspace is None:
        workspace = _scratch(stream, remainder_workspace(prob), q.device)
    ws_min = remainder_workspace(prob, 1)
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or workspace.numel() < ws_min:
        raise ValueError(f"workspace must be a uint8 device tensor of at least {ws_min} bytes")
    _check(load().sva_sparse_attention_remainder(
        ctypes.byref(prob), _ptr(q), _ptr(k), _ptr(v), _ptr(q_pool), _ptr(k_pool), _ptr(kv_idx), _ptr(kv_count),
        int(kmax), _ptr(workspace), int(workspace.numel()), _ptr(out), _ptr(lse), _stream(stream)),
        "sva_sparse_attention_remainder")
    _record(stream, q, k, v, q_pool, k_pool, kv_idx, kv_count, workspace, out, lse)
    return out, lse


def dense_attention(prob: Problem, q, k, v, out=None, want_lse: bool = False, lse=None,
                    stream=None) -> Tuple:
    torch = _torch()
    shp = _qkv_shape(prob)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, shp, n)
    out = _out_tensor(prob, q, out, stream)
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, shp[:3], dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, torch.float32, shp[:3], "lse")
    _check(load().sva_dense_attention(ctypes.byref(prob), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                      _ptr(lse), _stream(stream)), "sva_dense_attention")
    _record(stream, q, k, v, out, lse)
    return out, lse


# --------------------------------------------------------- fp8 (e4m3) attention

def fp8_padded_len(prob: Problem) -> int:
    out = ctypes.c_int32(0)
    _check(load().sva_fp8_padded_len(ctypes.byref(prob), ctypes.byref(out)), "sva_fp8_padded_len")
    return out.value


def fp8_code_dim(prob: Problem) -> int:
    out = ctypes.c_int32(0)
    _check(load().sva_fp8_code_dim(ctypes.byref(prob), ctypes.byref(out)), "sva_fp8_code_dim")
    return out.value


def _fp8_struct(t: dict) -> Fp8Tensors:
    return Fp8Tensors(*(_ptr(t.get(n)) for n in ("q8", "k8", "v8", "q_exp", "k_exp", "v_exp", "k_mean")))


def _need_fp8(prob: Problem, t: dict, need_mean: bool):
    torch = _torch()
    nb, npad, dp = num_blocks(prob), fp8_padded_len(prob), fp8_code_dim(prob)
    B, H, D = prob.batch, prob.heads, prob.head_dim
    _need(t["q8"], torch.uint8, (B, H, npad, dp), "q8")
    _need(t["k8"], torch.uint8, (B, H, npad, dp), "k8")
    _need(t["v8"], torch.uint8, (B, H, npad // 64, dp, 64), "v8")
    _need(t["q_exp"], torch.int32, (B, H, nb), "q_exp")
    _need(t["k_exp"], torch.int32, (B, H, nb), "k_exp")
    _need(t["v_exp"], torch.int32, (B, H, dp), "v_exp")
    if need_mean:
        _need(t["k_mean"], torch.bfloat16, (B, H, D), "k_mean")


def quantize_fp8(prob: Problem, q, k, v, out: Optional[dict] = None, stream=None) -> dict:
    """e4m3 codes and power-of-two exponents of Q, K (smoothed) and V
    (sva_quantize_fp8).  Returns {q8, k8, v8, q_exp, k_exp, v_exp, k_mean}."""
    torch = _torch()
    shp = _qkv_shape(prob)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, shp, n)
    if out is None:
        nb, npad, dp = num_blocks(prob), fp8_padded_len(prob), fp8_code_dim(prob)
        B, H, D = prob.batch, prob.heads, prob.head_dim
        dev = q.device
        out = {"q8": _output(stream, torch.empty, (B, H, npad, dp), dtype=torch.uint8, device=dev),
               "k8": _output(stream, torch.empty, (B, H, npad, dp), dtype=torch.uint8, device=dev),
               "v8": _output(stream, torch.empty, (B, H, npad // 64, dp, 64), dtype=torch.uint8, device=dev),
               "q_exp": _output(stream, torch.empty, (B, H, nb), dtype=torch.int32, device=dev),
               "k_exp": _output(stream, torch.empty, (B, H, nb), dtype=torch.int32, device=dev),
               "v_exp": _output(stream, torch.empty, (B, H, dp), dtype=torch.int32, device=dev),
               "k_mean": _output(stream, torch.empty, (B, H, D), dtype=torch.bfloat16, device=dev)}
    _need_fp8(prob, out, True)
    st = _fp8_struct(out)
    _check(load().sva_quantize_fp8(ctypes.byref(prob), _ptr(q), _ptr(k), _ptr(v), ctypes.byref(st),
                                   _stream(stream)), "sva_quantize_fp8")
    _record(stream, q, k, v, out)
    return out


def sparse_attention_fp8(prob: Problem, quant: dict, kv_idx, kv_count, out=None,
                         want_lse: bool = False, lse=None, stream=None) -> Tuple:
    """Block-sparse attention on the codes of quantize_fp8 (sva_sparse_attention_fp8)."""
    torch = _torch()
    nb = num_blocks(prob)
    shp = _qkv_shape(prob)
    _need_fp8(prob, quant, False)
    kmax = kv_idx.shape[-1]
    _need(kv_idx, torch.int32, (prob.batch, prob.heads, nb, kmax), "kv_idx")
    _need(kv_count, torch.int32, (prob.batch, prob.heads, nb), "kv_count")
    ref = quant["q8"]
    if out is None:
        dt = torch.float32 if prob.out_dtype == SVA_F32 else torch.bfloat16
        out = _output(stream, torch.empty, shp, dtype=dt, device=ref.device)
    _need(out, torch.float32 if prob.out_dtype == SVA_F32 else torch.bfloat16, shp, "out")
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, shp[:3], dtype=torch.float32, device=ref.device)
    if lse is not None:
        _need(lse, torch.float32, shp[:3], "lse")
    st = _fp8_struct(quant)
    _check(load().sva_sparse_attention_fp8(ctypes.byref(prob), ctypes.byref(st), _ptr(kv_idx),
                                           _ptr(kv_count), int(kmax), _ptr(out), _ptr(lse),
                                           _stream(stream)), "sva_sparse_attention_fp8")
    _record(stream, quant, kv_idx, kv_count, out, lse)
    return out, lse


def dense_attention_fp8(prob: Problem, quant: dict, out=None, want_lse: bool = False, lse=None,
                        stream=None) -> Tuple:
    """Every block kept, on the codes of quantize_fp8 (sva_dense_attention_fp8)."""
    torch = _torch()
    shp = _qkv_shape(prob)
    _need_fp8(prob, quant, False)
    ref = quant["q8"]
    dt = torch.float32 if prob.out_dtype == SVA_F32 else torch.bfloat16
    if out is None:
        out = _output(stream, torch.empty, shp, dtype=dt, device=ref.device)
    _need(out, dt, shp, "out")
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, shp[:3], dtype=torch.float32, device=ref.device)
    if lse is not None:
        _need(lse, torch.float32, shp[:3], "lse")
    st = _fp8_struct(quant)
    _check(load().sva_dense_attention_fp8(ctypes.byref(prob), ctypes.byref(st), _ptr(out), _ptr(lse),
                                          _stream(stream)), "sva_dense_attention_fp8")
    _record(stream, quant, out, lse)
    return out, lse


# ------------------------------------------------------------- token pruning

def tokens(batch: int, n_tokens: int, channels: int) -> Tokens:
    return Tokens(int(batch), int(n_tokens), int(channels))


def token_keep_count(t: Tokens, keep_ratio: float) -> int:
    out = ctypes.c_int32(0)
    _check(load().sva_token_keep_count(ctypes.byref(t), float(keep_ratio), ctypes.byref(out)),
           "sva_token_keep_count")
    return out.value


def token_select_workspace(t: Tokens) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sva_token_select_workspace(ctypes.byref(t), ctypes.byref(out)),
           "sva_token_select_workspace")
    return out.value


def token_select(x, keep_ratio: float, scores=None, kept_idx=None, kept_pos=None,
                 workspace=None, stream=None) -> Tuple:
    """feat_norm scores and kept tokens of hidden states x (bf16 [B, N, C]),
    sva_token_select: returns (scores float64 [B, N], kept_idx int32 [B, k]
    ascending, kept_pos int32 [B, N] with -1 for dropped tokens).  workspace:
    a uint8 device tensor of token_select_workspace bytes (allocated when
    None; pass one to reuse it)."""
    torch = _torch()
    if x.dim() != 3:
        raise ValueError("x must be [B, N, C]")
    B, N, C = x.shape
    t = tokens(B, N, C)
    k = token_keep_count(t, keep_ratio)
    _need(x, torch.bfloat16, (B, N, C), "x")
    if scores is None:
        scores = _output(stream, torch.empty, (B, N), dtype=torch.float64, device=x.device)
    else:
        _need(scores, torch.float64, (B, N), "scores")
    if kept_idx is None:
        kept_idx = _output(stream, torch.empty, (B, k), dtype=torch.int32, device=x.device)
    else:
        _need(kept_idx, torch.int32, (B, k), "kept_idx")
    if kept_pos is None:
        kept_pos = _output(stream, torch.empty, (B, N), dtype=torch.int32, device=x.device)
    else:
        _need(kept_pos, torch.int32, (B, N), "kept_pos")
    ws_bytes = token_select_workspace(t)
    if workspace is None:
        workspace = _scratch(stream, ws_bytes, x.device)
    if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous()
            and workspace.numel() * workspace.element_size() >= ws_bytes):
        raise ValueError(f"workspace must be a contiguous device tensor of >= {ws_bytes} bytes")
    _check(load().sva_token_select(ctypes.byref(t), float(keep_ratio), _ptr(x), _ptr(scores),
                                   _ptr(kept_idx), _ptr(kept_pos), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)),
           "sva_token_select")
    _record(stream, x, scores, kept_idx, kept_pos, workspace)
    return scores, kept_idx, kept_pos


def token_select_noalloc(x, keep_ratio: float, scores=None, kept_idx=None, kept_pos=None, stream=None) -> Tuple:
    """sva_token_select_noalloc: token_select with the library's static
    workspace (at most 16 batch entries; calls on one GPU must not overlap).
    Outputs are allocated here when not given; the library call itself
    allocates nothing."""
    torch = _torch()
    if x.dim() != 3:
        raise ValueError("x must be [B, N, C]")
    B, N, C = x.shape
    t = tokens(B, N, C)
    k = token_keep_count(t, keep_ratio)
    _need(x, torch.bfloat16, (B, N, C), "x")
    if scores is None:
        scores = _output(stream, torch.empty, (B, N), dtype=torch.float64, device=x.device)
    else:
        _need(scores, torch.float64, (B, N), "scores")
    if kept_idx is None:
        kept_idx = _output(stream, torch.empty, (B, k), dtype=torch.int32, device=x.device)
    else:
        _need(kept_idx, torch.int32, (B, k), "kept_idx")
    if kept_pos is None:
        kept_pos = _output(stream, torch.empty, (B, N), dtype=torch.int32, device=x.device)
    else:
        _need(kept_pos, torch.int32, (B, N), "kept_pos")
    _check(load().sva_token_select_noalloc(ctypes.byref(t), float(keep_ratio), _ptr(x), _ptr(scores),
                                           _ptr(kept_idx), _ptr(kept_pos), _stream(stream)),
           "sva_token_select_noalloc")
    _record(stream, x, scores, kept_idx, kept_pos)
    return scores, kept_idx, kept_pos


def token_gather(x, kept_idx, x_kept=None, stream=None):
    """x_kept[b, j] = x[b, kept_idx[b, j]] (sva_token_gather)."""
    torch = _torch()
    B, N, C = x.shape
    k = kept_idx.shape[1]
    _need(x, torch.bfloat16, (B, N, C), "x")
    _need(kept_idx, torch.int32, (B, k), "kept_idx")
    if x_kept is None:
        x_kept = _output(stream, torch.empty, (B, k, C), dtype=torch.bfloat16, device=x.device)
    else:
        _need(x_kept, torch.bfloat16, (B, k, C), "x_kept")
    _check(load().sva_token_gather(ctypes.byref(tokens(B, N, C)), k, _ptr(x), _ptr(kept_idx),
                                   _ptr(x_kept), _stream(stream)), "sva_token_gather")
    _record(stream, x, kept_idx, x_kept)
    return x_kept


def token_scatter(y_kept, kept_pos, base, out=None, stream=None):
    """out[b, n] = y_kept[b, kept_pos[b, n]] for kept tokens, base[b, n] for the
    others (sva_token_scatter); out may be base (in place)."""
    torch = _torch()
    B, N, C = base.shape
    k = y_kept.shape[1]
    _need(y_kept, torch.bfloat16, (B, k, C), "y_kept")
    _need(kept_pos, torch.int32, (B, N), "kept_pos")
    _need(base, torch.bfloat16, (B, N, C), "base")
    if out is None:
        out = _output(stream, torch.empty_like, base)
    else:
        _need(out, torch.bfloat16, (B, N, C), "out")
    _check(load().sva_token_scatter(ctypes.byref(tokens(B, N, C)), k, _ptr(y_kept), _ptr(kept_pos),
                                    _ptr(base), _ptr(out), _stream(stream)), "sva_token_scatter")
    _record(stream, y_kept, kept_pos, base, out)
    return out


# ------------------------------------- rotary positions, the key/value cache

# (As above, these calls' time is this module's own where tensors are small: a tensor that is
# as it should be passes one test, and what is wrong with another is found out afterwards.)

def _device() -> int:
    """The current device, on whose streams calls are launched."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getDevice", None)
    return raw() if raw is not None and torch.cuda.is_initialized() else torch.cuda.current_device()


def _stream_on(stream, dev: int):
    return _stream(stream) if stream is not None else _torch()._C._cuda_getCurrentRawStream(dev)


def _refuse(t, dtype, shape, name, dev=None):
    """Raises for a tensor that is not on the current device, or of another type or shape."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    dev = _device() if dev is None else dev
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _on_device(t, name):
    """A tensor on the current device; which device that is."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    dev = _device()
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")
    return dev


def _heads(t, dtype, shape, name, dev) -> Heads:
    """A tensor [B, H, N, D] with any strides, its channels contiguous."""
    if not (isinstance(t, _torch().Tensor) and t.dtype == dtype and t.shape == shape and t.get_device() == dev):
        _refuse(t, dtype, shape, name, dev)
    sb, sh, sn, sd = t.stride()
    if sd != 1 and shape[3] > 1:
        raise ValueError(f"{name}'s channels must be contiguous (stride 1), got stride {sd}")
    return Heads(t.data_ptr(), shape[1], sb, sh, sn)


def _plain(t, dtype, shape, name, dev) -> int:
    """A contiguous tensor's pointer."""
    if not (isinstance(t, _torch().Tensor) and t.dtype == dtype and t.shape == shape and t.get_device() == dev
            and t.is_contiguous()):
        _refuse(t, dtype, shape, name, dev)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows_of_ints(t, batch, columns, name, dev):
    """int32 [batch, columns] or [columns] (shared): its pointer and batch stride."""
    torch = _torch()
    if not (isinstance(t, torch.Tensor) and t.dtype == torch.int32 and t.get_device() == dev):
        _refuse(t, torch.int32, getattr(t, "shape", ()), name, dev)
    shape = t.shape
    if len(shape) == 2 and shape[0] == batch and shape[1] == columns:
        stride, step = t.stride()
    elif len(shape) == 1 and shape[0] == columns:
        step, stride = t.stride(0), 0
    else:
        raise ValueError(f"{name} must have shape {(batch, columns)} or {(columns,)}, got {tuple(shape)}")
    if step != 1 and columns > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return t.data_ptr(), stride


def _dtype_code(dtype, name):
    torch = _torch()
    if dtype == torch.bfloat16 or dtype == "bf16":
        return torch.bfloat16, SVA_BF16
    if dtype == torch.float32 or dtype in ("f32", "float32"):
        return torch.float32, SVA_F32
    raise TypeError(f"{name} must be bfloat16 or float32, got {dtype}")


def rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original_len: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0,
                       magnitude: float = 0.0) -> Tuple:
    """(list of rot_dim / 2 frequencies in radians per position, factor on cosine
    and sine), sva_rotary_frequencies.  scaling: "none", "linear", "ntk" or
    "yarn"; factor: how many times longer the contexts are; original_len: the
    trained one ("yarn")."""
    if scaling not in SVA_ROTARY_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(SVA_ROTARY_SCALINGS)}, got {scaling!r}")
    spec = RotarySpec(int(rot_dim), SVA_ROTARY_SCALINGS[scaling], float(base), float(factor), float(original_len),
                      float(beta_fast), float(beta_slow), float(magnitude))
    freq = (ctypes.c_double * max(1, int(rot_dim) // 2))()
    mag = ctypes.c_double()
    _check(load().sva_rotary_frequencies(ctypes.byref(spec), freq, ctypes.byref(mag)), "sva_rotary_frequencies")
    return list(freq), mag.value


def rotary_plan(head_dim: int, rot_dim: Optional[int] = None, layout: str = "half", base: float = 10000.0,
                scaling: str = "none", factor: float = 1.0, original_len: float = 0.0, beta_fast: float = 32.0,
                beta_slow: float = 1.0, magnitude: float = 0.0, device="cuda") -> dict:
    """What rotary() turns by, made once: {head_dim, rot_dim, layout, magnitude,
    freq (float64 [rot_dim / 2] on the device)}.  rot_dim: the channels turned,
    the first of each head (all when None); layout: "half" (pairs i, i + rot_dim/2)
    or "interleaved" (pairs 2i, 2i + 1); the rest as in rotary_frequencies."""
    if layout not in SVA_ROTARY_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(SVA_ROTARY_LAYOUTS)}, got {layout!r}")
    rot_dim = head_dim if rot_dim is None else rot_dim
    if rot_dim > head_dim:
        raise ValueError(f"rot_dim {rot_dim} exceeds head_dim {head_dim}")
    freq, mag = rotary_frequencies(rot_dim, base, scaling, factor, original_len, beta_fast, beta_slow, magnitude)
    torch = _torch()
    return {"head_dim": int(head_dim), "rot_dim": int(rot_dim), "layout": layout, "magnitude": mag,
            "freq": torch.tensor(freq, dtype=torch.float64, device=device)}


def rotary(plan: dict, positions, q, k=None, q_out=None, k_out=None, backward: bool = False, stream=None) -> Tuple:
    """Rotary positions of q [B, H, N, D] and, in the same launch, k [B, Hk, N, D]
    (bf16 or float32, any strides with contiguous channels: a slice of a fused
    projection is taken as it lies), sva_rotary.  positions: int32 [B, N], or [N]
    for all entries.  q_out / k_out may be q / k (in place).  backward: the
    transposed map, from gradients of the outputs to gradients of the inputs.
    Returns (q_out, k_out), k_out None without k."""
    torch = _torch()
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise ValueError("q must be a tensor [B, H, N, D]")
    shp = q.shape
    B, H, N, D = shp
    if D != plan["head_dim"]:
        raise ValueError(f"q has {D} channels, the plan {plan['head_dim']}")
    dt, code = _dtype_code(q.dtype, "q")
    dev = _on_device(q, "q")
    qi = _heads(q, dt, shp, "q", dev)
    if q_out is None:
        q_out = _output(stream, torch.empty_like, q)
    qo = _heads(q_out, dt, shp, "q_out", dev)
    ki = ko = None
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k must be a tensor [B, H, N, D]")
        shp = (B, k.shape[1], N, D)
        ki = _heads(k, dt, shp, "k", dev)
        if k_out is None:
            k_out = _output(stream, torch.empty_like, k)
        ko = _heads(k_out, dt, shp, "k_out", dev)
    elif k_out is not None:
        raise ValueError("k_out without k")
    freq, rot = plan["freq"], plan["rot_dim"]
    pos, pos_b = _rows_of_ints(positions, B, N, "positions", dev)
    prm = RotaryParams(B, N, D, rot, SVA_ROTARY_LAYOUTS[plan["layout"]], code, 1 if backward else 0, plan["magnitude"])
    _check(load().sva_rotary(prm, _plain(freq, torch.float64, (rot // 2,), "plan['freq']", dev), pos, pos_b, qi, qo, ki,
                             ko, _stream_on(stream, dev)), "sva_rotary")
    _record(stream, q, k, q_out, k_out, freq, positions)
    return q_out, k_out


def kv_cache(num_pages: int, kv_heads: int, head_dim: int, page_size: int = 64, fmt: str = "e4m3",
             device="cuda") -> dict:
    """An empty paged cache: {k, v: [num_pages, kv_heads, page_size, head_dim]
    codes (bfloat16, uint8 e4m3 bytes or int8, as fmt is "bf16", "e4m3" or
    "int8"), k_scale, v_scale: float32 [num_pages, kv_heads, page_size], None for
    bf16}.  Any tensors of these shapes and types are a cache."""
    torch = _torch()
    if fmt not in SVA_CACHE_FORMATS:
        raise ValueError(f"fmt must be one of {sorted(SVA_CACHE_FORMATS)}, got {fmt!r}")
    dt = {"bf16": torch.bfloat16, "e4m3": torch.uint8, "int8": torch.int8}[fmt]
    shp = (int(num_pages), int(kv_heads), int(page_size), int(head_dim))
    cache = {n: torch.zeros(shp, dtype=dt, device=device) for n in ("k", "v")}
    for n in ("k_scale", "v_scale"):
        cache[n] = None if fmt == "bf16" else torch.zeros(shp[:3], dtype=torch.float32, device=device)
    return cache


def _cache(c: dict, dev=None) -> Cache:
    torch = _torch()
    k, v = c["k"], c["v"]
    if dev is None:
        dev = _on_device(k, "cache['k']")
    dt = k.dtype
    fmt = 1 if dt == torch.uint8 else 2 if dt == torch.int8 else 0 if dt == torch.bfloat16 else None
    if fmt is None:
        raise TypeError(f"cache['k'] must be bfloat16, uint8 (e4m3) or int8, got {dt}")
    shp = k.shape
    if len(shp) != 4:
        raise ValueError("cache['k'] must be [pages, kv_heads, page_size, head_dim]")
    kp, vp = _plain(k, dt, shp, "cache['k']", dev), _plain(v, dt, shp, "cache['v']", dev)
    ks = vs = None
    if fmt:
        rows = shp[:3]
        ks = _plain(c["k_scale"], torch.float32, rows, "cache['k_scale']", dev)
        vs = _plain(c["v_scale"], torch.float32, rows, "cache['v_scale']", dev)
    return Cache(fmt, shp[0], shp[1], shp[2], shp[3], kp, vp, ks, vs)


def cache_write(cache: dict, k, v, slots, stream=None) -> dict:
    """Quantise the rows of k and v (bf16 or float32 [B, kv_heads, N, D], any
    strides with contiguous channels) into slots (int32 [B, N]; page * page_size +
    place; out of range: nothing is written; the others distinct),
    sva_cache_write.  Returns the cache."""
    torch = _torch()
    dev = _on_device(k, "k")
    st = _cache(cache, dev)
    if k.dim() != 4:
        raise ValueError("k must be a tensor [B, kv_heads, N, D]")
    dt, code = _dtype_code(k.dtype, "k")
    B, _, N, _ = k.shape
    shp = (B, st.kv_heads, N, st.head_dim)
    hk, hv = _heads(k, dt, shp, "k", dev), _heads(v, dt, shp, "v", dev)
    ptr, sb = _rows_of_ints(slots, B, N, "slots", dev)
    if B > 1 and slots.dim() == 1:
        raise ValueError("slots must be [B, N]: entries cannot share slots")
    _check(load().sva_cache_write(st, B, N, code, hk, hv, ptr, sb, _stream_on(stream, dev)), "sva_cache_write")
    if stream is not None:
        _record(stream, k, v, slots, *cache.values())
    return cache


def cache_read(cache: dict, slots, k=None, v=None, dtype="bf16", stream=None) -> Tuple:
    """The tokens at slots (int32 [B, N]; out of range: zeros) as K and V
    [B, kv_heads, N, D] of dtype ("bf16" or "f32"), sva_cache_read; contiguous
    where allocated here, as the whole-sequence operators take them."""
    torch = _torch()
    dev = _on_device(slots, "slots")
    st = _cache(cache, dev)
    if slots.dim() != 2:
        raise ValueError("slots must be a tensor [B, N]")
    B, N = slots.shape
    dt, code = _dtype_code(dtype, "dtype")
    shp = (B, st.kv_heads, N, st.head_dim)
    ptr, sb = _rows_of_ints(slots, B, N, "slots", dev)
    if k is None:
        k = _output(stream, torch.empty, shp, dtype=dt, device=slots.device)
    if v is None:
        v = _output(stream, torch.empty, shp, dtype=dt, device=slots.device)
    _check(load().sva_cache_read(st, B, N, code, ptr, sb, _heads(k, dt, shp, "k", dev), _heads(v, dt, shp, "v", dev),
                                 _stream_on(stream, dev)), "sva_cache_read")
    if stream is not None:
        _record(stream, k, v, slots, *cache.values())
    return k, v


def cache_attention_workspace(cache: dict, batch: int, heads: int, queries: int, max_pages: int) -> int:
    """Workspace bytes of cache_attention for B = batch, H = heads, T = queries and
    a page table of max_pages columns (sva_cache_attention_workspace)."""
    out = ctypes.c_size_t(0)
    _check(load().sva_cache_attention_workspace(_cache(cache), CacheQuery(batch, heads, queries, max_pages, 0.0, SVA_BF16),
                                                ctypes.byref(out)), "sva_cache_attention_workspace")
    return out.value


_workspace_bytes = {}      # sva_cache_attention_workspace by sizes


def cache_attention(cache: dict, q, page_table, lengths, k_new=None, v_new=None, mask=None, counts=None,
                    softmax_scale: float = 0.0, out_dtype="bf16", out=None, want_lse: bool = False, lse=None,
                    workspace=None, stream=None) -> Tuple:
    """Attention of T drafted tokens per entry (one in plain decoding), q bf16
    [B, H, T, D], over the cached tokens that page_table (int32 [B, max_pages]) and
    lengths (int32 [B]) name and over each other, sva_cache_attention.  k_new,
    v_new: bf16 [B, kv_heads, T, D]; mask: uint8 or bool [B, T, T] or [T, T], token
    t sees drafted token s where mask[b, t, s] is not zero (None: s <= t); counts:
    int32 [B], the drafted tokens an entry has (None: T).  q, k_new, v_new and out
    take any strides with contiguous channels that are multiples of 16 bytes; out
    is made like q, of out_dtype ("bf16" or "f32").  workspace: a uint8 device
    tensor of cache_attention_workspace bytes (allocated when None).  Returns
    (out, lse)."""
    torch = _torch()
    dev = _on_device(q, "q")
    st = _cache(cache, dev)
    shp = q.shape
    if len(shp) != 4:
        raise ValueError("q must be a tensor [B, H, T, D]")
    B, H, T, D = shp
    if D != st.head_dim:
        raise ValueError(f"q has {D} channels, the cache {st.head_dim}")
    bf16, i32 = torch.bfloat16, torch.int32
    hq = _heads(q, bf16, shp, "q", dev)
    lens = _plain(lengths, i32, (B,), "lengths", dev)
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be a tensor [B, max_pages]")
    pages = page_table.shape[1]
    table = _plain(page_table, i32, (B, pages), "page_table", dev)
    hk = hv = mk = cnt = None
    if (k_new is None) != (v_new is None):
        raise ValueError("k_new and v_new go together")
    if k_new is not None:
        new = (B, st.kv_heads, T, D)
        hk, hv = _heads(k_new, bf16, new, "k_new", dev), _heads(v_new, bf16, new, "v_new", dev)
    mask_b = 0
    if mask is not None:
        if k_new is None:
            raise ValueError("mask without drafted keys")
        _on_device(mask, "mask")
        if mask.dtype != torch.uint8 and mask.dtype != torch.bool:
            raise TypeError(f"mask must be uint8 or bool, got {mask.dtype}")
        if mask.shape != (B, T, T) and mask.shape != (T, T):
            raise ValueError(f"mask must have shape {(B, T, T)} or {(T, T)}, got {tuple(mask.shape)}")
        strides = mask.stride()
        if T > 1 and (strides[-1] != 1 or strides[-2] != T):
            raise ValueError("mask's last two dimensions must be contiguous")
        mask_b = strides[0] if len(strides) == 3 else 0
        mk = mask.data_ptr()
    if counts is not None:
        cnt = _plain(counts, i32, (B,), "counts", dev)
    if out is None:
        dt, code = _dtype_code(out_dtype, "out_dtype")
        out = _output(stream, torch.empty_like, q, dtype=dt)
    else:
        dt, code = _dtype_code(out.dtype, "out")
    ho = _heads(out, dt, shp, "out", dev)
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, (B, H, T), dtype=torch.float32, device=q.device)
    lp = None if lse is None else _plain(lse, torch.float32, (B, H, T), "lse", dev)
    qry = CacheQuery(B, H, T, pages, float(softmax_scale), code)
    lib = load()
    ws_ptr, ws_bytes = None, 0
    if workspace is None:
        sizes = (B, H, T, pages, st.kv_heads, st.page_size, D)
        ws_bytes = _workspace_bytes.get(sizes)
        if ws_bytes is None:
            need = ctypes.c_size_t(0)
            _check(lib.sva_cache_attention_workspace(st, qry, need), "sva_cache_attention_workspace")
            if len(_workspace_bytes) > 4096:
                _workspace_bytes.clear()
            ws_bytes = _workspace_bytes[sizes] = need.value
        if ws_bytes:
            workspace = _scratch(stream, ws_bytes, q.device)
            ws_ptr = workspace.data_ptr()
    else:
        ws_bytes = workspace.numel()
        ws_ptr = _plain(workspace, torch.uint8, (ws_bytes,), "workspace", dev)
    _check(lib.sva_cache_attention(st, qry, hq, table, lens, hk, hv, mk, mask_b, cnt, ws_ptr, ws_bytes, ho, lp,
                                   _stream_on(stream, dev)), "sva_cache_attention")
    if stream is not None:
        _record(stream, q, page_table, lengths, k_new, v_new, mask, counts, workspace, out, lse, *cache.values())
    return out, lse
