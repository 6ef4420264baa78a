"""Binding of what stands around self-attention in a denoiser's layer: rotary positions
on several axes, layer norm, cross attention, and their gradients.  Argument
marshalling only, as in _lib.py, whose conventions hold here: streams, outputs and
workspaces, errors.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

from . import _lib
from ._lib import (SVA_BF16, SVA_F32, SVA_POSITIONS_F32, SVA_POSITIONS_I32, SVA_ROTARY_LAYOUTS, SVA_ROTARY_SCALINGS, Cross,
                   LayerNormParams, Positions, RotarySpec, Rows, _check, _dtype_code, _heads, _on_device, _output, _plain,
                   _ptr, _record, _refuse, _rotary_tensors, _scratch, _stream_on, _torch)


# -------------------------------------------------- rotary positions on several axes

def _per_axis(x, count, name):
    """A value for every axis: the one given, or count of them."""
    if isinstance(x, (tuple, list)):
        if len(x) != count:
            raise ValueError(f"{name} must be one value or {count}, got {len(x)}")
        return [float(v) for v in x]
    return [float(x)] * count


def rotary_axes_plan(head_dim: int, sections, layout: str = "half", base=10000.0, scaling: str = "none", factor=1.0,
                     original_len=0.0, beta_fast: float = 32.0, beta_slow: float = 1.0, magnitude: float = 0.0,
                     device="cuda") -> dict:
    """What rotary_axes() turns by, made once (sva_rotary_axes_frequencies): a rotary_plan
    with "axes" and "axis" (int32 [rot_dim / 2] on the device, the axis of each pair; a
    program may lay out its own).  sections: pairs of each axis, one axis after the other
    (time, height, width), each with frequencies base^(-j / its pairs); base, factor and
    original_len: one value, or one per axis; the rest as in rotary_frequencies."""
    if layout not in SVA_ROTARY_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(SVA_ROTARY_LAYOUTS)}, got {layout!r}")
    if scaling not in SVA_ROTARY_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(SVA_ROTARY_SCALINGS)}, got {scaling!r}")
    sections = [int(n) for n in sections]
    count, pairs = len(sections), sum(sections)
    if count < 1 or min(sections) < 1:
        raise ValueError(f"sections must be numbers of pairs, got {sections}")
    if 2 * pairs > head_dim:
        raise ValueError(f"sections turn {2 * pairs} channels, more than head_dim {head_dim}")
    specs = (RotarySpec * count)(*(RotarySpec(2 * n, SVA_ROTARY_SCALINGS[scaling], b, f, o, float(beta_fast),
                                              float(beta_slow), float(magnitude))
                                   for n, b, f, o in zip(sections, _per_axis(base, count, "base"),
                                                         _per_axis(factor, count, "factor"),
                                                         _per_axis(original_len, count, "original_len"))))
    freq, axis, mag = (ctypes.c_double * pairs)(), (ctypes.c_int32 * pairs)(), ctypes.c_double()
    _check(_lib.load().sva_rotary_axes_frequencies(specs, count, freq, axis, ctypes.byref(mag)), "sva_rotary_axes_frequencies")
    torch = _torch()
    return {"head_dim": int(head_dim), "rot_dim": 2 * pairs, "layout": layout, "magnitude": mag.value, "axes": count,
            "freq": torch.tensor(list(freq), dtype=torch.float64, device=device),
            "axis": torch.tensor(list(axis), dtype=torch.int32, device=device)}


def rotary_axes(plan: dict, positions, q, k=None, q_out=None, k_out=None, backward: bool = False, stream=None) -> Tuple:
    """rotary() with positions on several axes, sva_rotary_axes: int32 or float32
    [B, N, axes] of any strides, or [N, axes] for all entries."""
    torch = _torch()
    dev, prm, q_out, k_out, (qi, qo, ki, ko) = _rotary_tensors(plan, q, k, q_out, k_out, backward, stream)
    freq, axis, count = plan["freq"], plan["axis"], plan["axes"]
    _on_device(positions, "positions")
    if positions.dtype != torch.int32 and positions.dtype != torch.float32:
        raise TypeError(f"positions must be int32 or float32, got {positions.dtype}")
    want = (prm.batch, prm.tokens, count)
    if positions.shape != want and positions.shape != want[1:]:
        raise ValueError(f"positions must have shape {want} or {want[1:]}, got {tuple(positions.shape)}")
    strides = positions.stride()
    # a dimension of one has no stride
    pos = Positions(positions.data_ptr(), SVA_POSITIONS_F32 if positions.dtype == torch.float32 else SVA_POSITIONS_I32, count,
                    strides[0] if len(strides) == 3 and prm.batch > 1 else 0, strides[-2] if prm.tokens > 1 else 0,
                    strides[-1] if count > 1 else 0)
    pairs = (prm.rot_dim // 2,)
    _check(_lib.load().sva_rotary_axes(prm, _plain(freq, torch.float64, pairs, "plan['freq']", dev),
                                  _plain(axis, torch.int32, pairs, "plan['axis']", dev), pos, qi, qo, ki, ko,
                                  _stream_on(stream, dev)), "sva_rotary_axes")
    _record(stream, q, k, q_out, k_out, freq, axis, positions)
    return q_out, k_out


# --------------------------------------------------- layer norm, cross attention

def _rows(t, dtype, shape, name, dev) -> Rows:
    """A tensor [B, N, C] with any strides, its channels contiguous."""
    if not (isinstance(t, _torch().Tensor) and t.dtype == dtype and t.shape == shape and t.get_device() == dev):
        _refuse(t, dtype, shape, name, dev)
    sb, sn, sc = t.stride()
    if sc != 1 and shape[2] > 1:
        raise ValueError(f"{name}'s channels must be contiguous (stride 1), got stride {sc}")
    return Rows(t.data_ptr(), sb, sn)


def _norm_rows(t, B, C, name, dev):
    """weight or bias, [C] or [B, C]: 1 for a row per entry, and the stride of entries."""
    if not (isinstance(t, _torch().Tensor) and t.get_device() == dev):
        _on_device(t, name)
    shape, strides = t.shape, t.stride()
    if len(shape) == 2 and shape[0] == B and shape[1] == C:
        per, stride = 1, strides[0]
    elif len(shape) == 1 and shape[0] == C:
        per = stride = 0
    else:
        raise ValueError(f"{name} must have shape {(C,)} or {(B, C)}, got {tuple(shape)}")
    if C > 1 and strides[-1] != 1:
        raise ValueError(f"{name}'s channels must be contiguous")
    return per, stride


def _norm_weights(weight, bias, B, C, dev):
    """weight and bias, [C] or [B, C] and of one type: (pointers, type code, per entry, strides)."""
    if weight is None and bias is None:
        return None, None, SVA_F32, 0, 0, 0
    per_w = per_b = None
    w_s = b_s = 0
    if weight is not None:
        per_w, w_s = _norm_rows(weight, B, C, "weight", dev)
    if bias is not None:
        per_b, b_s = _norm_rows(bias, B, C, "bias", dev)
    if weight is not None and bias is not None:
        if weight.dtype != bias.dtype:
            raise TypeError(f"weight and bias must have one type, got {weight.dtype} and {bias.dtype}")
        if per_w != per_b:
            raise ValueError("weight and bias must both be [C] or both [B, C]")
    _, code = _dtype_code((bias if weight is None else weight).dtype, "weight and bias")
    return _ptr(weight), _ptr(bias), code, per_b if weight is None else per_w, w_s, b_s


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, unit_offset: bool = False, y=None, want_stats: bool = False,
               mean=None, rstd=None, stream=None) -> Tuple:
    """Layer norm over the channels of x [B, N, C] (bf16 or float32, any strides with
    contiguous channels), sva_layer_norm.  weight and bias: bf16 or float32 [C], or [B, C]
    with a row per batch entry (adaptive norm; a slice of a modulation is taken as it
    lies); unit_offset: the factor is 1 + weight.  y may be x.  want_stats: mean and rstd,
    float32 [B, N], which layer_norm_backward takes.  Returns (y, mean, rstd)."""
    torch = _torch()
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError("x must be a tensor [B, N, C]")
    shp = x.shape
    B, N, C = shp
    dt, code = _dtype_code(x.dtype, "x")
    dev = _on_device(x, "x")
    w, b, w_code, per, w_s, b_s = _norm_weights(weight, bias, B, C, dev)
    rx = _rows(x, dt, shp, "x", dev)
    if y is None:
        y = _output(stream, torch.empty_like, x)
    if want_stats and mean is None:
        mean = _output(stream, torch.empty, (B, N), dtype=torch.float32, device=x.device)
    if want_stats and rstd is None:
        rstd = _output(stream, torch.empty, (B, N), dtype=torch.float32, device=x.device)
    mp = None if mean is None else _plain(mean, torch.float32, (B, N), "mean", dev)
    rp = None if rstd is None else _plain(rstd, torch.float32, (B, N), "rstd", dev)
    prm = LayerNormParams(B, N, C, code, w_code, per, 1 if unit_offset else 0, w_s, b_s, float(eps))
    _check(_lib.load().sva_layer_norm(prm, rx, w, b, _rows(y, dt, shp, "y", dev), mp, rp, _stream_on(stream, dev)),
           "sva_layer_norm")
    if stream is not None:
        _record(stream, x, weight, bias, y, mean, rstd)
    return y, mean, rstd


def layer_norm_backward_workspace(batch: int, n_tokens: int, channels: int, per_entry: bool = False) -> int:
    """Workspace bytes of layer_norm_backward (sva_layer_norm_backward_workspace)."""
    out = ctypes.c_size_t(0)
    prm = LayerNormParams(batch, n_tokens, channels, SVA_BF16, SVA_F32, 1 if per_entry else 0, 0, 0, 0, 1.0)
    _check(_lib.load().sva_layer_norm_backward_workspace(prm, ctypes.byref(out)), "sva_layer_norm_backward_workspace")
    return out.value


_norm_bytes = {}           # workspace bytes by sizes


def layer_norm_backward(dy, x, mean, rstd, weight=None, unit_offset: bool = False, dx=None, want_weight: bool = True,
                        per_entry: Optional[bool] = None, dweight=None, dbias=None, workspace=None, stream=None) -> Tuple:
    """Gradients of layer_norm, sva_layer_norm_backward: dx like x from dy (both [B, N, C]
    of one type), x, and mean and rstd as layer_norm gave them; weight and unit_offset as
    there.  want_weight: the sums for weight and bias, float32 [C], or [B, C] where weight
    is [B, C] (per_entry: says so where there is no weight, but a bias).  dx may be dy or
    x.  workspace: a uint8 device tensor of layer_norm_backward_workspace bytes (allocated
    when None).  Returns (dx, dweight, dbias)."""
    torch = _torch()
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError("x must be a tensor [B, N, C]")
    shp = x.shape
    B, N, C = shp
    dt, code = _dtype_code(x.dtype, "x")
    dev = _on_device(x, "x")
    w, _, w_code, per, w_s, _ = _norm_weights(weight, None, B, C, dev)
    if weight is None:
        per = 1 if per_entry else 0
    elif per_entry is not None and bool(per) != bool(per_entry):
        raise ValueError(f"per_entry does not fit weight of shape {tuple(weight.shape)}")
    rg, rx = _rows(dy, dt, shp, "dy", dev), _rows(x, dt, shp, "x", dev)
    if dx is None:
        dx = _output(stream, torch.empty_like, x)
    ro = _rows(dx, dt, shp, "dx", dev)
    sums = (B, C) if per else (C,)
    if want_weight and dweight is None:
        dweight = _output(stream, torch.empty, sums, dtype=torch.float32, device=x.device)
    if want_weight and dbias is None:
        dbias = _output(stream, torch.empty, sums, dtype=torch.float32, device=x.device)
    prm = LayerNormParams(B, N, C, code, w_code, per, 1 if unit_offset else 0, w_s, 0, 1.0)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        ws_bytes = workspace.numel()
        ws_ptr = _plain(workspace, torch.uint8, (ws_bytes,), "workspace", dev)
    elif dweight is not None or dbias is not None:
        # with shared weights, entries whose rows follow each other are one, and need the sums of one
        one = (not per and rg.stride_b == N * rg.stride_n and rx.stride_b == N * rx.stride_n
               and ro.stride_b == N * ro.stride_n and B * N < 1 << 31)
        key = (1, B * N, C, 0) if one else (B, N, C, per)
        ws_bytes = _norm_bytes.get(key)
        if ws_bytes is None:
            if len(_norm_bytes) > 4096:
                _norm_bytes.clear()
            ws_bytes = _norm_bytes[key] = layer_norm_backward_workspace(*key)
        if ws_bytes:
            workspace = _scratch(stream, ws_bytes, x.device)
            ws_ptr = workspace.data_ptr()
    _check(_lib.load().sva_layer_norm_backward(
        prm, rg, rx, w, _plain(mean, torch.float32, (B, N), "mean", dev), _plain(rstd, torch.float32, (B, N), "rstd", dev),
        ws_ptr, ws_bytes, ro,
        None if dweight is None else _plain(dweight, torch.float32, sums, "dweight", dev),
        None if dbias is None else _plain(dbias, torch.float32, sums, "dbias", dev), _stream_on(stream, dev)),
        "sva_layer_norm_backward")
    if stream is not None:
        _record(stream, dy, x, mean, rstd, weight, dx, dweight, dbias, workspace)
    return dx, dweight, dbias


def cross_attention_workspace(batch: int, heads: int, kv_heads: int, queries: int, keys: int, head_dim: int,
                              masked: bool = False, backward: bool = False) -> int:
    """Workspace bytes of cross_attention, or of cross_attention_backward, with a mask or
    without (sva_cross_attention_workspace, sva_cross_attention_backward_workspace)."""
    out = ctypes.c_size_t(0)
    name = "sva_cross_attention_backward_workspace" if backward else "sva_cross_attention_workspace"
    _check(getattr(_lib.load(), name)(Cross(batch, heads, kv_heads, queries, keys, head_dim, 0.0), 1 if masked else 0,
                                 ctypes.byref(out)), name)
    return out.value


def _cross(q, k, lengths, mask, softmax_scale):
    """What both cross-attention calls check first: sizes, and which keys are hidden."""
    torch = _torch()
    dev = _on_device(q, "q")
    if q.dim() != 4:
        raise ValueError("q must be a tensor [B, H, N, D]")
    if not isinstance(k, torch.Tensor) or k.dim() != 4:
        raise ValueError("k must be a tensor [B, kv_heads, M, D]")
    B, H, N, D = q.shape
    _, kv, M, _ = k.shape
    lens = None if lengths is None else _plain(lengths, torch.int32, (B,), "lengths", dev)
    mk, mask_b = None, 0
    if mask is not None:
        _on_device(mask, "mask")
        if mask.dtype != torch.uint8 and mask.dtype != torch.bool:
            raise TypeError(f"mask must be uint8 or bool, got {mask.dtype}")
        if mask.shape != (B, M) and mask.shape != (M,):
            raise ValueError(f"mask must have shape {(B, M)} or {(M,)}, got {tuple(mask.shape)}")
        if M > 1 and mask.stride(-1) != 1:
            raise ValueError("mask's rows must be contiguous")
        mk, mask_b = mask.data_ptr(), mask.stride(0) if mask.dim() == 2 and B > 1 else 0
    return dev, Cross(B, H, kv, N, M, D, float(softmax_scale)), (B, H, N, D), (B, kv, M, D), lens, mk, mask_b


def _cross_workspace(workspace, stream, x, dev, backward):
    """The workspace of a call: (tensor or None, pointer, bytes)."""
    if workspace is not None:
        n = workspace.numel()
        return workspace, _plain(workspace, _torch().uint8, (n,), "workspace", dev), n
    sizes, masked, device = x
    key = (backward, masked, sizes.batch, sizes.heads, sizes.kv_heads, sizes.queries, sizes.keys, sizes.head_dim)
    need = _cross_bytes.get(key)
    if need is None:
        if len(_cross_bytes) > 4096:
            _cross_bytes.clear()
        need = _cross_bytes[key] = cross_attention_workspace(*key[2:], masked=masked, backward=backward)
    if need == 0:
        return None, None, 0
    workspace = _scratch(stream, need, device)
    return workspace, workspace.data_ptr(), need


_cross_bytes = {}          # workspace bytes by sizes


def cross_attention(q, k, v, lengths=None, mask=None, softmax_scale: float = 0.0, out=None, want_lse: bool = False, lse=None,
                    workspace=None, stream=None) -> Tuple:
    """softmax(c q k^T) v of q bf16 [B, H, N, D] over an encoder's states k, v bf16
    [B, kv_heads, M, D] (N and M from one on; H a multiple of kv_heads),
    sva_cross_attention.  lengths: int32 [B], an entry's keys; mask: uint8 or bool [B, M]
    or [M], nonzero where a key is seen.  q, k, v and out take any strides with contiguous
    channels that are multiples of 16 bytes; out is made like q, and shares no byte with what
    is read (slices of one projection may interleave).  want_lse: float32 [B, H, N], which
    cross_attention_backward takes.  workspace: a uint8 device tensor of
    cross_attention_workspace bytes (allocated when None).  Returns (out, lse)."""
    torch = _torch()
    dev, prm, rows, states, lens, mk, mask_b = _cross(q, k, lengths, mask, softmax_scale)
    bf16 = torch.bfloat16
    hq, hk, hv = _heads(q, bf16, rows, "q", dev), _heads(k, bf16, states, "k", dev), _heads(v, bf16, states, "v", dev)
    if out is None:
        out = _output(stream, torch.empty_like, q)
    if want_lse and lse is None:
        lse = _output(stream, torch.empty, rows[:3], dtype=torch.float32, device=q.device)
    lp = None if lse is None else _plain(lse, torch.float32, rows[:3], "lse", dev)
    ho = _heads(out, bf16, rows, "out", dev)
    workspace, ws_ptr, ws_bytes = _cross_workspace(workspace, stream, (prm, mk is not None, q.device), dev, False)
    _check(_lib.load().sva_cross_attention(prm, hq, hk, hv, lens, mk, mask_b, ws_ptr, ws_bytes, ho, lp, _stream_on(stream, dev)),
           "sva_cross_attention")
    if stream is not None:
        _record(stream, q, k, v, lengths, mask, workspace, out, lse)
    return out, lse


def cross_attention_backward(dout, q, k, v, out, lse, lengths=None, mask=None, softmax_scale: float = 0.0, dq=None, dk=None,
                             dv=None, workspace=None, stream=None) -> Tuple:
    """Gradients of q, k and v, like them, from dout (like out), with out and lse as
    cross_attention gave them for the same arguments, sva_cross_attention_backward.  dq, dk
    and dv share no byte with each other or with what is read.  workspace: a uint8 device tensor of cross_attention_workspace(..., backward=True)
    bytes (allocated when None).  Returns (dq, dk, dv)."""
    torch = _torch()
    dev, prm, rows, states, lens, mk, mask_b = _cross(q, k, lengths, mask, softmax_scale)
    bf16 = torch.bfloat16
    hg = _heads(dout, bf16, rows, "dout", dev)
    hq, hk, hv = _heads(q, bf16, rows, "q", dev), _heads(k, bf16, states, "k", dev), _heads(v, bf16, states, "v", dev)
    ho = _heads(out, bf16, rows, "out", dev)
    lp = _plain(lse, torch.float32, rows[:3], "lse", dev)
    dq = _output(stream, torch.empty_like, q) if dq is None else dq
    dk = _output(stream, torch.empty_like, k) if dk is None else dk
    dv = _output(stream, torch.empty_like, v) if dv is None else dv
    gq, gk, gv = _heads(dq, bf16, rows, "dq", dev), _heads(dk, bf16, states, "dk", dev), _heads(dv, bf16, states, "dv", dev)
    workspace, ws_ptr, ws_bytes = _cross_workspace(workspace, stream, (prm, mk is not None, q.device), dev, True)
    _check(_lib.load().sva_cross_attention_backward(prm, hg, hq, hk, hv, ho, lp, lens, mk, mask_b, ws_ptr, ws_bytes, gq, gk, gv,
                                               _stream_on(stream, dev)), "sva_cross_attention_backward")
    if stream is not None:
        _record(stream, dout, q, k, v, out, lse, lengths, mask, workspace, dq, dk, dv)
    return dq, dk, dv
