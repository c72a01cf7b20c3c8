"""The operators of a denoiser block around the hybrid attention, on torch CUDA tensors: layer norm, rotary positions with several axes,
gated feed-forward, forward and backward.  Each is one call of the library (include/hf.h) on the current stream; outputs and workspaces
come from torch's allocator.  There is no fallback: a tensor the library does not take raises.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as hf

_TYPES = {torch.bfloat16: hf.HF_BF16, torch.float16: hf.HF_F16, torch.float32: hf.HF_F32}
_PAIRINGS = {"adjacent": hf.HF_PAIRS_ADJACENT, "halves": hf.HF_PAIRS_HALVES}
_ACTS = {"silu": hf.HF_ACT_SILU, "gelu_tanh": hf.HF_ACT_GELU_TANH}


def _want(ok: bool, text: str):
    if not ok:
        raise ValueError(text)


def _cuda(name, t, shape=None, dtype=None):
    if not t.is_cuda:
        raise ValueError(f"{name} is not on a CUDA device")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


def _type(name, t):
    if t.dtype not in _TYPES:
        raise ValueError(f"{name}: {t.dtype} is not taken")
    return _TYPES[t.dtype]


def _rows(name, t):
    """t as rows of its last axis: (rows, width, elements between rows).  Raises where the rows have no common stride."""
    width = t.shape[-1]
    if t.dim() == 2:
        if width > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}: the last axis has to be contiguous")
        return t.shape[0], width, t.stride(0) if t.shape[0] > 1 else max(width, 1)
    if t.dim() == 1:
        return _rows(name, t[None])
    try:
        v = t.view(-1, width) if t.numel() else t.reshape(-1, width) if width else t.new_empty(0, 0)
    except RuntimeError:
        raise ValueError(f"{name}: the leading axes have no common stride") from None
    return _rows(name, v)


# ------------------------------------------------------------------------------------------------ layer norm
def _norm_shape(x, weight, bias, eps, weight_offset, rows_per_group):
    rows, width, stride = _rows("x", x)
    _want(width >= 1, "x has rows of no elements")
    _cuda("x", x)
    s = hf.hf_norm_shape(type=_type("x", x), width=width, rows=rows, x_stride=stride, y_stride=width, dx_stride=width,
                         rows_per_group=rows_per_group, param_stride=width, weight_offset=weight_offset, eps=eps)
    s.param_type = s.type
    groups = -(-rows // rows_per_group) if rows_per_group > 0 else 1
    for name, p in (("weight", weight), ("bias", bias)):
        if p is None:
            continue
        _cuda(name, p)
        _want(p.dtype in (x.dtype, torch.float32), f"{name} is {p.dtype}: x's type or float32 is taken")
        n, w, ps = _rows(name, p)
        _want(w == width and n == groups, f"{name} has shape {tuple(p.shape)}: {groups} rows of {width} are taken")
        s.param_type = _TYPES[p.dtype]
        s.param_stride = ps
    if weight is not None and bias is not None:
        _want(weight.dtype == bias.dtype, "weight and bias have different types")
        _want(groups == 1 or _rows("weight", weight)[2] == _rows("bias", bias)[2], "weight and bias have different strides")
    return s, groups


def layer_norm(x, weight=None, bias=None, eps=1e-6, weight_offset=0.0, rows_per_group=0):
    """y = (x - mean) * rstd * (weight_offset + weight) + bias over the last axis; returns (y, mean, rstd), the last two float32 [rows].
    x: bf16, f16 or f32 [..., width], rows with one common stride.  weight, bias: [width] or [1, width]; with rows_per_group > 0
    [groups, width], row r of x taking row r // rows_per_group (slices of a modulation tensor are fine); x's type or float32; or None."""
    s, _ = _norm_shape(x, weight, bias, eps, weight_offset, rows_per_group)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = torch.empty(s.rows, dtype=torch.float32, device=x.device)
    rstd = torch.empty(s.rows, dtype=torch.float32, device=x.device)
    hf.hf_layer_norm(s, x, weight, bias, y, mean, rstd)
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, weight_offset=0.0, rows_per_group=0):
    """Gradients of `layer_norm`: (dx in x's type, dweight, dbias float32 [groups, width]).  mean, rstd: as the forward returned them."""
    s, groups = _norm_shape(x, weight, None, 0.0, weight_offset, rows_per_group)
    _cuda("dy", dy, x.shape, x.dtype)
    _cuda("mean", mean, (s.rows,), torch.float32)
    _cuda("rstd", rstd, (s.rows,), torch.float32)
    _want(mean.is_contiguous() and rstd.is_contiguous(), "mean and rstd have to be contiguous")
    s.y_stride = _rows("dy", dy)[2]
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    d_params = torch.empty((2, groups, s.width), dtype=torch.float32, device=x.device)
    dw, db = d_params.unbind(0)
    ws = torch.empty(hf.hf_layer_norm_workspace(s), dtype=torch.uint8, device=x.device)
    hf.hf_layer_norm_backward(s, dy, x, mean, rstd, weight, dx, dw, db, ws)
    return dx, dw, db


# ------------------------------------------------------------------------------------------------ rotary positions
def _rope(tensors, pos, tables, pairing, inverse):
    """tensors: (x, y, rotate) with x, y [batch, tokens, heads, head_dim] of any strides, features contiguous."""
    cos, sin, extents, pairs = tables
    x = tensors[0][0]
    B, T, _, d = x.shape
    axes = len(pairs)
    _want(1 <= axes <= 4 and len(extents) == axes, "one to four axes, an extent and a number of pairs for each")
    _want(pairing in _PAIRINGS, f"pairing {pairing!r} unknown")
    n = sum(e * p for e, p in zip(extents, pairs))
    for name, t in (("cos", cos), ("sin", sin)):
        _cuda(name, t, (n,), torch.float32)
        _want(t.is_contiguous(), f"{name} has to be contiguous")
    _cuda("pos", pos, None, torch.int32)
    _want(tuple(pos.shape) in ((T, axes), (1, T, axes), (B, T, axes)) and pos.is_contiguous(),
          f"pos has shape {tuple(pos.shape)}: contiguous [{T}, {axes}] or [{B}, {T}, {axes}] is taken")
    s = hf.hf_rope_shape(type=_type("x", x), batch=B, tokens=T, head_dim=d, axes=axes, pairing=_PAIRINGS[pairing], inverse=inverse,
                         pos_batch=T * axes if pos.dim() == 3 and pos.shape[0] == B and B > 1 else 0)
    s.pairs[:axes] = pairs
    s.extent[:axes] = extents
    arr = (hf.hf_rope_tensor * len(tensors))()
    for a, (x, y, rotate) in zip(arr, tensors):
        xs, ys = x.stride(), y.stride()
        _want((xs[3] == 1 and ys[3] == 1) or d == 1, "the features of a head have to be contiguous")
        a.x, a.y, a.heads, a.rotate = x.data_ptr(), y.data_ptr(), x.shape[2], rotate
        a.x_batch, a.x_token, a.x_head = xs[0], xs[1], xs[2]
        a.y_batch, a.y_token, a.y_head = ys[0], ys[1], ys[2]
    hf.hf_rope_axes(s, arr, len(tensors), cos, sin, pos)


def rope_axes(x, pos, tables, out=None, pairing="adjacent", inverse=False):
    """x [batch, tokens, heads, head_dim] (any strides, features contiguous) turned by its tokens' positions.  pos: int32 [tokens, axes]
    or [batch, tokens, axes]; tables: (cos, sin, extents, pairs per axis) as `rope.axis_tables` forms cos and sin, on the device.
    out: a tensor of x's shape and type with strides of its own, or x itself; None: a new one.  inverse: the backward pass."""
    _want(x.dim() == 4, "x is [batch, tokens, heads, head_dim]")
    _cuda("x", x)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _cuda("out", out, x.shape, x.dtype)
    _rope([(x, out, 1)], pos, tables, pairing, inverse)
    return out


def split_heads_rope(qkv, heads, kv_heads, pos, tables, pairing="adjacent"):
    """Rows of a fused projection [batch, tokens, (heads + 2 kv_heads) * head_dim] (row stride free) -> q, k, v [batch, heads, tokens, head_dim]
    as the hybrid attention takes them, q and k turned by their positions, in one launch."""
    _want(qkv.dim() == 3, "qkv is [batch, tokens, (heads + 2 kv_heads) * head_dim]")
    B, T, W = qkv.shape
    _want(heads >= 1 and kv_heads >= 1 and W % (heads + 2 * kv_heads) == 0, f"{W} columns do not divide into {heads} + 2 x {kv_heads} heads")
    _cuda("qkv", qkv)
    _want(W == 1 or qkv.stride(2) == 1, "the last axis has to be contiguous")
    d = W // (heads + 2 * kv_heads)
    q = torch.empty((B, heads, T, d), dtype=qkv.dtype, device=qkv.device)
    k = torch.empty((B, kv_heads, T, d), dtype=qkv.dtype, device=qkv.device)
    v = torch.empty((B, kv_heads, T, d), dtype=qkv.dtype, device=qkv.device)
    xq, xk, xv = qkv.unflatten(2, (heads + 2 * kv_heads, d)).split([heads, kv_heads, kv_heads], dim=2)
    _rope([(xq, q.transpose(1, 2), 1), (xk, k.transpose(1, 2), 1), (xv, v.transpose(1, 2), 0)], pos, tables, pairing, 0)
    return q, k, v


def split_heads_rope_backward(dq, dk, dv, pos, tables, pairing="adjacent"):
    """Gradient of `split_heads_rope` with respect to the rows: [batch, tokens, (heads + 2 kv_heads) * head_dim], contiguous."""
    B, H, T, d = dq.shape
    KV = dk.shape[1]
    for name, t, h in (("dq", dq, H), ("dk", dk, KV), ("dv", dv, KV)):
        _cuda(name, t, (B, h, T, d), dq.dtype)
    out = torch.empty((B, T, (H + 2 * KV) * d), dtype=dq.dtype, device=dq.device)
    yq, yk, yv = out.view(B, T, H + 2 * KV, d).split([H, KV, KV], dim=2)
    _rope([(dq.transpose(1, 2), yq, 1), (dk.transpose(1, 2), yk, 1), (dv.transpose(1, 2), yv, 0)], pos, tables, pairing, 1)
    return out


# ------------------------------------------------------------------------------------------------ gated feed-forward
def _ff_shape(x, w_gate, w_up, w_down, act):
    rows, width, stride = _rows("x", x)
    _want(act in _ACTS, f"act {act!r} unknown")
    _cuda("x", x)
    hidden, out_width = w_gate.shape[0], w_down.shape[0]
    for name, w, shape in (("w_gate", w_gate, (hidden, width)), ("w_up", w_up, (hidden, width)), ("w_down", w_down, (out_width, hidden))):
        _cuda(name, w, shape, x.dtype)
        _want(w.is_contiguous(), f"{name} has to be contiguous")
    return hf.hf_ff_shape(type=_type("x", x), act=_ACTS[act], rows=rows, width=width, hidden=hidden, out_width=out_width, x_stride=stride,
                          y_stride=out_width)


def gated_ff(x, w_gate, w_up, w_down, act="silu", save=False):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T.  x bf16 or f16 [..., width], rows with one common stride; w_gate, w_up [hidden, width],
    w_down [out_width, hidden] contiguous; act "silu" or "gelu_tanh".  save: returns (y, gate, up), the last two [rows, hidden] for
    `gated_ff_backward`; otherwise y alone."""
    s = _ff_shape(x, w_gate, w_up, w_down, act)
    y = torch.empty(x.shape[:-1] + (s.out_width,), dtype=x.dtype, device=x.device)
    gate = torch.empty((s.rows, s.hidden), dtype=x.dtype, device=x.device) if save else None
    up = torch.empty((s.rows, s.hidden), dtype=x.dtype, device=x.device) if save else None
    ws = torch.empty(hf.hf_gated_ff_workspace(s, 0), dtype=torch.uint8, device=x.device)
    hf.hf_gated_ff(s, x, w_gate, w_up, w_down, y, gate, up, ws)
    return (y, gate, up) if save else y


def gated_ff_backward(dy, x, w_gate, w_up, w_down, gate, up, act="silu"):
    """Gradients of `gated_ff`: (dx, dw_gate, dw_up, dw_down) in x's type.  gate, up: as the forward returned them."""
    s = _ff_shape(x, w_gate, w_up, w_down, act)
    _cuda("dy", dy, tuple(x.shape[:-1]) + (s.out_width,), x.dtype)
    for name, t in (("gate", gate), ("up", up)):
        _cuda(name, t, (s.rows, s.hidden), x.dtype)
        _want(t.is_contiguous(), f"{name} has to be contiguous")
    s.y_stride = _rows("dy", dy)[2]
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dwg, dwu, dwd = torch.empty_like(w_gate), torch.empty_like(w_up), torch.empty_like(w_down)
    ws = torch.empty(hf.hf_gated_ff_workspace(s, 1), dtype=torch.uint8, device=x.device)
    hf.hf_gated_ff_backward(s, dy, x, w_gate, w_up, w_down, gate, up, dx, dwg, dwu, dwd, ws)
    return dx, dwg, dwu, dwd
