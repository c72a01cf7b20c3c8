"""The operators of a denoiser block around the hybrid attention, on torch CUDA tensors: layer norm, rotary positions with several axes (with norms of
q and k or without), gated feed-forward, linear layers with their epilogue, forward and backward.  Each is one call of the library (include/hf.h) on the current stream; outputs and workspaces
come from torch's allocator.  There is no fallback: a tensor the library does not take raises.

Where gradients are recorded and an input needs one, `layer_norm`, `rope_axes`, `split_heads_rope`, `split_heads_norm_rope`, `gated_ff` and `linear` are part of torch's
graph, their backward passes the `*_backward` calls below (which may also be called by hand); a second derivative raises.

The short calls are bound by the host, so the way to the library is kept short: the shapes are packed as the bytes of the C structures,
tensors are asked for nothing twice, and outputs come from the cheapest of torch's ways to make one (empty_like and new_empty with plain
numbers take 1.4 us, torch.empty with a type and a device 2.4, a view 1.1).
"""
from __future__ import annotations

import functools
import struct

import torch
from torch.autograd.function import once_differentiable

from . import binding as hf

_TYPES = {torch.bfloat16: hf.HF_BF16, torch.float16: hf.HF_F16, torch.float32: hf.HF_F32}
_PAIRINGS = {"adjacent": hf.HF_PAIRS_ADJACENT, "halves": hf.HF_PAIRS_HALVES}
_OVERS = {"head": hf.HF_NORM_OVER_HEAD, "width": hf.HF_NORM_OVER_WIDTH}
_ACTS = {"silu": hf.HF_ACT_SILU, "gelu_tanh": hf.HF_ACT_GELU_TANH}
_LINEAR_ACTS = {None: hf.HF_ACT_NONE, **_ACTS}
_NORM = struct.Struct("@3i6q2f").pack                       # hf_norm_shape
_ROPE = struct.Struct("@5i4i4i2iq").pack                    # hf_rope_shape
_ROPE_TENSOR = struct.Struct("@2P6q2i").pack                # hf_rope_tensor
_ROPE_TENSORS = struct.Struct("@2P6q2i2P6q2i2P6q2i").pack   # three of them
_HEADS = struct.Struct("@18if5q").pack                      # hf_heads_shape
_HEADS_TENSORS = struct.Struct("@P3qP3qP3q").pack           # three hf_heads_tensor
_FF = struct.Struct("@2iq3i2q").pack                        # hf_ff_shape
_LINEAR = struct.Struct("@5i6q").pack                       # hf_linear_shape
_F32, _I32 = torch.float32, torch.int32
_empty_like, _empty_strided = torch.empty_like, torch.empty_strided
_lib, _stream, _check = hf.lib, hf._stream, hf._check
_recording = torch.is_grad_enabled


try:
    _device = torch._C._cuda_getDevice          # torch's raw getter, which has no public name, spares a microsecond a call
except AttributeError:
    _device = torch.cuda.current_device


def _fail(text: str):
    raise ValueError(text)


def _here(name, t, dev):
    if t.get_device() != dev:
        _fail(f"{name} is on {t.device}, not on the current CUDA device")


def _current(name, t) -> int:
    """The current device, which t has to be on."""
    dev = t.get_device()
    if dev < 0 or dev != _device():
        _fail(f"{name} is on {t.device}, not on the current CUDA device")
    return dev


def _like(name, t, dev, shape, dtype):
    """t on the device, of that shape and type."""
    if t.get_device() != dev or t.dtype != dtype or t.shape != shape:
        _here(name, t, dev)
        _fail(f"{name} is {t.dtype} {tuple(t.shape)}: {dtype} {tuple(shape)} is taken")


def _dense(name, t, dev, shape, dtype):
    _like(name, t, dev, shape, dtype)
    if not t.is_contiguous():
        _fail(f"{name} has to be contiguous")


def _rows(name, t):
    """t as rows of its last axis: (rows, width, elements between rows).  Raises where the rows have no common stride."""
    shape = t.shape
    n = len(shape)
    if n == 0:
        _fail(f"{name} has no axes")
    width = shape[-1]
    if n != 2:
        rows = t.numel() // width if width else 0
        if t.is_contiguous():
            return rows, width, width
        try:
            t = t.view(rows, width)
        except RuntimeError:
            _fail(f"{name}: the leading axes have no common stride")
    rows = t.shape[0]
    stride, one = t.stride()
    if one != 1 and width > 1 and rows:         # (of no rows: whatever it says)
        _fail(f"{name}: the last axis has to be contiguous")
    return rows, width, stride if rows > 1 else width


# ------------------------------------------------------------------------------------------------ layer norm
def _norm_param(name, p, dev, dtype, width, groups):
    """Type and row stride of weight or bias."""
    shape, kind = p.shape, p.dtype
    if kind != dtype and kind != _F32:
        _fail(f"{name} is {kind}: x's type or float32 is taken")
    if p.get_device() != dev:
        _here(name, p, dev)
    if shape != (groups, width) and not (groups == 1 and shape == (width,)):
        _fail(f"{name} has shape {tuple(shape)}: {groups} rows of {width} are taken")
    strides = p.stride()
    if strides[-1] != 1 and width > 1:
        _fail(f"{name}: the last axis has to be contiguous")
    return kind, strides[0] if groups > 1 else width


def _norm_params(weight, bias, dev, dtype, width, groups):
    """Type and row stride of weight and bias together."""
    if weight is None and bias is None:
        return _TYPES[dtype], width
    if weight is None:
        kind, stride = _norm_param("bias", bias, dev, dtype, width, groups)
        return _TYPES[kind], stride
    kind, stride = _norm_param("weight", weight, dev, dtype, width, groups)
    if bias is not None and _norm_param("bias", bias, dev, dtype, width, groups) != (kind, stride):
        _fail("weight and bias differ in their type or their stride")
    return _TYPES[kind], stride


def _norm_type(x, width):
    if x.dtype not in _TYPES:
        _fail(f"x is {x.dtype}: bfloat16, float16 and float32 are taken")
    if width < 1:
        _fail("x has rows of no elements")
    return _TYPES[x.dtype]


def layer_norm(x, weight=None, bias=None, eps=1e-6, weight_offset=0.0, rows_per_group=0):
    """y = (x - mean) * rstd * (weight_offset + weight) + bias over the last axis; returns (y, mean, rstd), the last two float32 [rows].
    x: bf16, f16 or f32 [..., width], rows with one common stride.  weight, bias: [width] or [1, width]; with rows_per_group > 0
    [groups, width], row r of x taking row r // rows_per_group (slices of a modulation tensor are fine); x's type or float32; or None."""
    if _recording() and (x.requires_grad or weight is not None and weight.requires_grad or bias is not None and bias.requires_grad):
        return _LayerNorm.apply(x, weight, bias, eps, weight_offset, rows_per_group)
    dev = _current("x", x)
    rows, width, stride = _rows("x", x)
    t = _norm_type(x, width)
    pt, ps = _norm_params(weight, bias, dev, x.dtype, width, -(-rows // rows_per_group) if rows_per_group > 0 else 1)
    y = _empty_like(x) if stride == width else x.new_empty(x.shape)
    mean = _empty_strided((rows,), (1,), dtype=_F32, device=x.device)
    rstd = _empty_like(mean)
    status = _lib().hf_layer_norm(_NORM(t, pt, width, rows, stride, width, width, rows_per_group, ps, weight_offset, eps), x.data_ptr(),
                                  weight.data_ptr() if weight is not None else None, bias.data_ptr() if bias is not None else None,
                                  y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _stream())
    if status:
        _check(status)
    return y, mean, rstd


@functools.lru_cache(maxsize=256)
def _norm_workspace(dev, shape):
    return hf.hf_layer_norm_workspace(shape)


def layer_norm_backward(dy, x, mean, rstd, weight=None, weight_offset=0.0, rows_per_group=0):
    """Gradients of `layer_norm`: (dx in x's type, dweight, dbias float32 [groups, width]).  mean, rstd: as the forward returned them."""
    dev = _current("x", x)
    rows, width, stride = _rows("x", x)
    t = _norm_type(x, width)
    groups = -(-rows // rows_per_group) if rows_per_group > 0 else 1
    pt, ps = _norm_params(weight, None, dev, x.dtype, width, groups)
    _like("dy", dy, dev, x.shape, x.dtype)
    _dense("mean", mean, dev, (rows,), _F32)
    _dense("rstd", rstd, dev, (rows,), _F32)
    dx = _empty_like(x) if stride == width else x.new_empty(x.shape)
    dw = mean.new_empty(groups, width)
    db = _empty_like(dw)
    shape = _NORM(t, pt, width, rows, stride, _rows("dy", dy)[2], width, rows_per_group, ps, weight_offset, 0.0)
    ws = mean.new_empty(_norm_workspace(dev, shape) // 4)
    status = _lib().hf_layer_norm_backward(shape, dy.data_ptr(), x.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                           weight.data_ptr() if weight is not None else None, dx.data_ptr(), dw.data_ptr(), db.data_ptr(),
                                           ws.data_ptr(), _stream())
    if status:
        _check(status)
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, weight_offset, rows_per_group):
        y, mean, rstd = layer_norm(x, weight, bias, eps, weight_offset, rows_per_group)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias, ctx.args = None if bias is None else (bias.shape, bias.dtype), (weight_offset, rows_per_group)
        ctx.mark_non_differentiable(mean, rstd)
        ctx.set_materialize_grads(False)
        return y, mean, rstd

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, _mean, _rstd):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(dy.contiguous(), x, mean, rstd, weight, *ctx.args)
        return (dx, None if weight is None else dw.view(weight.shape).to(weight.dtype),
                None if ctx.bias is None else db.view(ctx.bias[0]).to(ctx.bias[1]), None, None, None)


# ------------------------------------------------------------------------------------------------ rotary positions
def _rope(x, B, T, d, tensors, n, pos, tables, pairing, inverse, dev):
    """tensors: the bytes of n hf_rope_tensor."""
    cos, sin, extents, pairs = tables
    axes = len(pairs)
    if not (1 <= axes <= 4 and len(extents) == axes):
        _fail("one to four axes, an extent and a number of pairs for each")
    if pairing not in _PAIRINGS:
        _fail(f"pairing {pairing!r} unknown")
    if x.dtype not in _TYPES:
        _fail(f"{x.dtype}: bfloat16, float16 and float32 are taken")
    n_entries = 0
    for e, p in zip(extents, pairs):
        n_entries += e * p
    if not (cos.dtype is _F32 and sin.dtype is _F32 and cos.get_device() == dev == sin.get_device() and cos.is_contiguous()
            and sin.is_contiguous() and cos.shape == (n_entries,) == sin.shape):
        _dense("cos", cos, dev, (n_entries,), _F32)
        _dense("sin", sin, dev, (n_entries,), _F32)
    shape = pos.shape
    if shape != (T, axes) and shape != (1, T, axes) and shape != (B, T, axes):
        _fail(f"pos has shape {tuple(shape)}: [{T}, {axes}] or [{B}, {T}, {axes}] is taken")
    if pos.dtype is not _I32 or pos.get_device() != dev or not pos.is_contiguous():
        _dense("pos", pos, dev, shape, _I32)
    rest = (0,) * (4 - axes)
    status = _lib().hf_rope_axes(_ROPE(_TYPES[x.dtype], B, T, d, axes, *pairs, *rest, *extents, *rest, _PAIRINGS[pairing], inverse,
                                       T * axes if B > 1 and len(shape) == 3 and shape[0] == B else 0), tensors, n, cos.data_ptr(), sin.data_ptr(),
                                 pos.data_ptr(), _stream())
    if status:
        _check(status)


def rope_axes(x, pos, tables, out=None, pairing="adjacent", inverse=False):
    """x [batch, tokens, heads, head_dim] (any strides, features contiguous) turned by its tokens' positions.  pos: int32 [tokens, axes]
    or [batch, tokens, axes]; tables: (cos, sin, extents, pairs per axis) as `rope.axis_tables` forms cos and sin, on the device.
    out: a tensor of x's shape and type with strides of its own, or x itself; None: a new one.  inverse: the backward pass."""
    if _recording() and (x.requires_grad or out is not None and out.requires_grad):
        if out is not None:
            _fail("out is not taken where gradients are recorded")
        return _RopeAxes.apply(x, pos, tables, pairing, inverse)
    dev = _current("x", x)
    if x.dim() != 4:
        _fail("x is [batch, tokens, heads, head_dim]")
    if out is None:
        out = x.new_empty(x.shape)
    else:
        _like("out", out, dev, x.shape, x.dtype)
    B, T, H, d = x.shape
    xb, xt, xh, x1 = x.stride()
    yb, yt, yh, y1 = out.stride()
    if (x1 != 1 or y1 != 1) and d > 1:
        _fail("the features of a head have to be contiguous")
    _rope(x, B, T, d, _ROPE_TENSOR(x.data_ptr(), out.data_ptr(), xb, xt, xh, yb, yt, yh, H, 1), 1, pos, tables, pairing, inverse, dev)
    return out


def split_heads_rope(qkv, heads, kv_heads, pos, tables, pairing="adjacent"):
    """Rows of a fused projection [batch, tokens, (heads + 2 kv_heads) * head_dim] (row stride free) -> q, k, v [batch, heads, tokens, head_dim]
    as the hybrid attention takes them, q and k turned by their positions, in one launch."""
    if _recording() and qkv.requires_grad:
        return _SplitHeadsRope.apply(qkv, heads, kv_heads, pos, tables, pairing)
    dev = _current("qkv", qkv)
    if qkv.dim() != 3:
        _fail("qkv is [batch, tokens, (heads + 2 kv_heads) * head_dim]")
    B, T, W = qkv.shape
    if heads < 1 or kv_heads < 1 or W % (heads + 2 * kv_heads):
        _fail(f"{W} columns do not divide into {heads} + 2 x {kv_heads} heads")
    xb, xt, one = qkv.stride()
    if one != 1 and W > 1:
        _fail("qkv: the last axis has to be contiguous")
    d = W // (heads + 2 * kv_heads)
    q = qkv.new_empty(B, heads, T, d)
    k = qkv.new_empty(B, kv_heads, T, d)
    v = _empty_like(k)
    x, td, e = qkv.data_ptr(), T * d, qkv.element_size()
    de, kv_batch = d * e, kv_heads * td
    _rope(qkv, B, T, d, _ROPE_TENSORS(x, q.data_ptr(), xb, xt, d, heads * td, d, td, heads, 1,
                                      x + heads * de, k.data_ptr(), xb, xt, d, kv_batch, d, td, kv_heads, 1,
                                      x + (heads + kv_heads) * de, v.data_ptr(), xb, xt, d, kv_batch, d, td, kv_heads, 0),
          3, pos, tables, pairing, 0, dev)
    return q, k, v


def split_heads_rope_backward(dq, dk, dv, pos, tables, pairing="adjacent"):
    """Gradient of `split_heads_rope` with respect to the rows: [batch, tokens, (heads + 2 kv_heads) * head_dim], contiguous."""
    dev = _current("dq", dq)
    if dq.dim() != 4 or dk.dim() != 4:
        _fail("dq, dk, dv are [batch, heads, tokens, head_dim]")
    B, H, T, d = dq.shape
    KV = dk.shape[1]
    _like("dk", dk, dev, (B, KV, T, d), dq.dtype)
    _like("dv", dv, dev, (B, KV, T, d), dq.dtype)
    W, e = (H + 2 * KV) * d, dq.element_size()
    out = dq.new_empty(B, T, W)
    at, parts = out.data_ptr(), b""
    for t, h, rotate in ((dq, H, 1), (dk, KV, 1), (dv, KV, 0)):
        xb, xh, xt, one = t.stride()
        if one != 1 and d > 1:
            _fail("the features of a head have to be contiguous")
        parts += _ROPE_TENSOR(t.data_ptr(), at, xb, xt, xh, T * W, W, d, h, rotate)
        at += h * d * e
    _rope(dq, B, T, d, parts, 3, pos, tables, pairing, 1, dev)
    return out


def _features_dense(t):
    """t with the features of a head contiguous; its other axes may lie as they do.  (A copy: `contiguous` keeps an expanded tensor of no elements as it is.)"""
    return t if t.stride(-1) == 1 else t.clone(memory_format=torch.contiguous_format)


class _RopeAxes(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, tables, pairing, inverse):
        cos, sin, *sizes = tables
        ctx.save_for_backward(pos, cos, sin)
        ctx.args = sizes, pairing, inverse
        return rope_axes(x, pos, tables, None, pairing, inverse)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        pos, cos, sin = ctx.saved_tensors
        sizes, pairing, inverse = ctx.args
        return rope_axes(_features_dense(dy), pos, (cos, sin, *sizes), None, pairing, not inverse), None, None, None, None


class _SplitHeadsRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, heads, kv_heads, pos, tables, pairing):
        cos, sin, *sizes = tables
        ctx.save_for_backward(pos, cos, sin)
        ctx.args = sizes, pairing
        return split_heads_rope(qkv, heads, kv_heads, pos, tables, pairing)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        pos, cos, sin = ctx.saved_tensors
        sizes, pairing = ctx.args
        return (split_heads_rope_backward(_features_dense(dq), _features_dense(dk), _features_dense(dv), pos, (cos, sin, *sizes), pairing),
                None, None, None, None, None)


# ------------------------------------------------------------------------------------------------ norms of q and k, with the rotation
def _norm_rope(qkv, heads, kv_heads, q_weight, k_weight, pos, tables, eps, over, pairing, grad_strides):
    """(device, batch, tokens, head_dim, the packed hf_heads_shape, cos, sin) of checked operands."""
    dev = _current("qkv", qkv)
    if qkv.dim() != 3:
        _fail("qkv is [batch, tokens, (heads + 2 kv_heads) * head_dim]")
    B, T, W = qkv.shape
    if heads < 1 or kv_heads < 1 or W % (heads + 2 * kv_heads):
        _fail(f"{W} columns do not divide into {heads} + 2 x {kv_heads} heads")
    xb, xt, one = qkv.stride()
    if one != 1 and W > 1:
        _fail("qkv: the last axis has to be contiguous")
    d = W // (heads + 2 * kv_heads)
    cos, sin, extents, pairs = tables
    axes = len(pairs)
    if not (1 <= axes <= 4 and len(extents) == axes):
        _fail("one to four axes, an extent and a number of pairs for each")
    if pairing not in _PAIRINGS:
        _fail(f"pairing {pairing!r} unknown")
    if over not in _OVERS:
        _fail(f"over {over!r} unknown")
    dtype = qkv.dtype
    if dtype not in _TYPES:
        _fail(f"qkv is {dtype}: bfloat16, float16 and float32 are taken")
    n_entries = 0
    for e, p in zip(extents, pairs):
        n_entries += e * p
    if not (cos.dtype is _F32 and sin.dtype is _F32 and cos.get_device() == dev == sin.get_device() and cos.is_contiguous()
            and sin.is_contiguous() and cos.shape == (n_entries,) == sin.shape):
        _dense("cos", cos, dev, (n_entries,), _F32)
        _dense("sin", sin, dev, (n_entries,), _F32)
    shape = pos.shape
    if shape != (T, axes) and shape != (1, T, axes) and shape != (B, T, axes):
        _fail(f"pos has shape {tuple(shape)}: [{T}, {axes}] or [{B}, {T}, {axes}] is taken")
    if pos.dtype is not _I32 or pos.get_device() != dev or not pos.is_contiguous():
        _dense("pos", pos, dev, shape, _I32)
    kind = dtype
    if q_weight is not None or k_weight is not None:
        kind = (k_weight if q_weight is None else q_weight).dtype
        if kind != dtype and kind != _F32:
            _fail(f"the weights are {kind}: qkv's type or float32 is taken")
        if q_weight is not None:
            _dense("q_weight", q_weight, dev, (d if over == "head" else heads * d,), kind)
        if k_weight is not None:
            _dense("k_weight", k_weight, dev, (d if over == "head" else kv_heads * d,), kind)
    rest = (0,) * (4 - axes)
    return dev, B, T, d, _HEADS(_TYPES[dtype], _TYPES[kind], B, T, d, heads, kv_heads, axes, *pairs, *rest, *extents, *rest, _PAIRINGS[pairing], _OVERS[over],
                                eps, T * axes if B > 1 and len(shape) == 3 and shape[0] == B else 0, xb, xt, *grad_strides), cos, sin


def split_heads_norm_rope(qkv, heads, kv_heads, q_weight, k_weight, pos, tables, eps=1e-6, over="head", pairing="adjacent"):
    """`split_heads_rope` of a block with norms of q and k, in one launch: before the rotation q and k are multiplied by 1 / sqrt(mean x^2 + eps), the
    mean over a head (over "head") or over all heads of the token ("width"), and by a weight, [head_dim] or [heads * head_dim] (k: kv_heads), of
    qkv's type or float32, or None."""
    if _recording() and (qkv.requires_grad or q_weight is not None and q_weight.requires_grad or k_weight is not None and k_weight.requires_grad):
        return _SplitHeadsNormRope.apply(qkv, heads, kv_heads, q_weight, k_weight, pos, tables, eps, over, pairing)
    dev, B, T, d, shape, cos, sin = _norm_rope(qkv, heads, kv_heads, q_weight, k_weight, pos, tables, eps, over, pairing, (0, 0))
    q = qkv.new_empty(B, heads, T, d)
    k = qkv.new_empty(B, kv_heads, T, d)
    v = _empty_like(k)
    td = T * d
    status = _lib().hf_split_heads_norm_rope(shape, qkv.data_ptr(), q_weight.data_ptr() if q_weight is not None else None,
                                             k_weight.data_ptr() if k_weight is not None else None, cos.data_ptr(), sin.data_ptr(), pos.data_ptr(),
                                             _HEADS_TENSORS(q.data_ptr(), heads * td, d, td, k.data_ptr(), kv_heads * td, d, td, v.data_ptr(), kv_heads * td, d, td),
                                             _stream())
    if status:
        _check(status)
    return q, k, v


@functools.lru_cache(maxsize=256)
def _norm_rope_workspace(dev, shape):
    return hf.hf_split_heads_norm_rope_workspace(shape)


def split_heads_norm_rope_backward(dq, dk, dv, qkv, q_weight, k_weight, pos, tables, eps=1e-6, over="head", pairing="adjacent"):
    """Gradients of `split_heads_norm_rope`: (dqkv contiguous, dq_weight, dk_weight float32).  dq, dk, dv: any strides with the features of a head contiguous."""
    if dq.dim() != 4 or dk.dim() != 4 or qkv.dim() != 3:
        _fail("dq, dk, dv are [batch, heads, tokens, head_dim], qkv [batch, tokens, (heads + 2 kv_heads) * head_dim]")
    W = qkv.shape[-1]
    dev, B, T, d, shape, cos, sin = _norm_rope(qkv, dq.shape[1], dk.shape[1], q_weight, k_weight, pos, tables, eps, over, pairing, (qkv.shape[1] * W, W))
    H, KV = dq.shape[1], dk.shape[1]
    _like("dq", dq, dev, (B, H, T, d), qkv.dtype)
    _like("dk", dk, dev, (B, KV, T, d), qkv.dtype)
    _like("dv", dv, dev, (B, KV, T, d), qkv.dtype)
    parts = ()
    for t in (dq, dk, dv):
        xb, xh, xt, one = t.stride()
        if one != 1 and d > 1:
            _fail("the features of a head have to be contiguous")
        parts += (t.data_ptr(), xb, xt, xh)
    out = qkv.new_empty(B, T, W)
    dqw = _empty_strided((d if over == "head" else H * d,), (1,), dtype=_F32, device=qkv.device)
    dkw = dqw.new_empty(d if over == "head" else KV * d)
    ws = dqw.new_empty(_norm_rope_workspace(dev, shape) // 4)
    status = _lib().hf_split_heads_norm_rope_backward(shape, _HEADS_TENSORS(*parts), qkv.data_ptr(), q_weight.data_ptr() if q_weight is not None else None,
                                                      k_weight.data_ptr() if k_weight is not None else None, cos.data_ptr(), sin.data_ptr(),
                                                      pos.data_ptr(), out.data_ptr(), dqw.data_ptr(), dkw.data_ptr(), ws.data_ptr(), _stream())
    if status:
        _check(status)
    return out, dqw, dkw


class _SplitHeadsNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, heads, kv_heads, q_weight, k_weight, pos, tables, eps, over, pairing):
        cos, sin, *sizes = tables
        ctx.save_for_backward(qkv, q_weight, k_weight, pos, cos, sin)
        ctx.args = sizes, eps, over, pairing
        return split_heads_norm_rope(qkv, heads, kv_heads, q_weight, k_weight, pos, tables, eps, over, pairing)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        qkv, q_weight, k_weight, pos, cos, sin = ctx.saved_tensors
        sizes, eps, over, pairing = ctx.args
        dqkv, dqw, dkw = split_heads_norm_rope_backward(_features_dense(dq), _features_dense(dk), _features_dense(dv), qkv, q_weight, k_weight, pos,
                                                        (cos, sin, *sizes), eps, over, pairing)
        return (dqkv, None, None, None if q_weight is None else dqw.to(q_weight.dtype), None if k_weight is None else dkw.to(k_weight.dtype),
                None, None, None, None, None)


# ------------------------------------------------------------------------------------------------ gated feed-forward
def _ff_operands(x, w_gate, w_up, w_down, act):
    """(device, type, rows, width, hidden, out_width, row stride of x) of checked operands."""
    dev = _current("x", x)
    rows, width, stride = _rows("x", x)
    if act not in _ACTS:
        _fail(f"act {act!r} unknown")
    if w_gate.dim() != 2 or w_down.dim() != 2:
        _fail("the weights are matrices")
    dtype, hidden, out_width = x.dtype, w_gate.shape[0], w_down.shape[0]
    if dtype not in _TYPES:
        _fail(f"x is {dtype}: bfloat16 and float16 are taken")
    if not (w_gate.dtype is dtype and w_up.dtype is dtype and w_down.dtype is dtype and w_gate.shape == (hidden, width) == w_up.shape
            and w_down.shape == (out_width, hidden) and w_gate.get_device() == dev == w_up.get_device() and w_down.get_device() == dev
            and w_gate.is_contiguous() and w_up.is_contiguous() and w_down.is_contiguous()):
        _dense("w_gate", w_gate, dev, (hidden, width), dtype)
        _dense("w_up", w_up, dev, (hidden, width), dtype)
        _dense("w_down", w_down, dev, (out_width, hidden), dtype)
    return dev, _TYPES[dtype], rows, width, hidden, out_width, stride


@functools.lru_cache(maxsize=256)
def _ff_workspace(dev, shape, backward):
    return hf.hf_gated_ff_workspace(shape, backward)


def gated_ff(x, w_gate, w_up, w_down, act="silu", save=False):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T.  x bf16 or f16 [..., width], rows with one common stride; w_gate, w_up [hidden, width],
    w_down [out_width, hidden] contiguous; act "silu" or "gelu_tanh".  save: returns (y, gate, up), the last two [rows, hidden] for
    `gated_ff_backward`; otherwise y alone.  act * up is rounded to x's type between the products: in float16 it ends at 65504."""
    if _recording() and (x.requires_grad or w_gate.requires_grad or w_up.requires_grad or w_down.requires_grad):
        return _GatedFF.apply(x, w_gate, w_up, w_down, act, save)
    dev, t, rows, width, hidden, out_width, stride = _ff_operands(x, w_gate, w_up, w_down, act)
    y = _empty_like(x) if out_width == width == stride else x.new_empty(x.shape[:-1] + (out_width,))
    gate = x.new_empty(rows, hidden) if save else None
    up = _empty_like(gate) if save else None
    shape = _FF(t, _ACTS[act], rows, width, hidden, out_width, stride, out_width)
    ws = x.new_empty(_ff_workspace(dev, shape, 0) // 2)
    status = _lib().hf_gated_ff(shape, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), y.data_ptr(),
                                gate.data_ptr() if save else None, up.data_ptr() if save else None, ws.data_ptr(), _stream())
    if status:
        _check(status)
    return (y, gate, up) if save else y


def gated_ff_backward(dy, x, w_gate, w_up, w_down, gate, up, act="silu"):
    """Gradients of `gated_ff`: (dx, dw_gate, dw_up, dw_down) in x's type.  gate, up: as the forward returned them.  The projections' gradients
    are rounded to x's type on the way: in float16 dy wants a scale that keeps them above 6e-5."""
    dev, t, rows, width, hidden, out_width, stride = _ff_operands(x, w_gate, w_up, w_down, act)
    _like("dy", dy, dev, x.shape[:-1] + (out_width,), x.dtype)
    _dense("gate", gate, dev, (rows, hidden), x.dtype)
    _dense("up", up, dev, (rows, hidden), x.dtype)
    dx = _empty_like(x) if stride == width else x.new_empty(x.shape)
    dwg, dwu, dwd = _empty_like(w_gate), _empty_like(w_up), _empty_like(w_down)
    shape = _FF(t, _ACTS[act], rows, width, hidden, out_width, stride, _rows("dy", dy)[2])
    ws = x.new_empty(_ff_workspace(dev, shape, 1) // 2)
    status = _lib().hf_gated_ff_backward(shape, dy.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(),
                                         gate.data_ptr(), up.data_ptr(), dx.data_ptr(), dwg.data_ptr(), dwu.data_ptr(), dwd.data_ptr(),
                                         ws.data_ptr(), _stream())
    if status:
        _check(status)
    return dx, dwg, dwu, dwd


class _GatedFF(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act, save):
        y, gate, up = gated_ff(x, w_gate, w_up, w_down, act, True)
        ctx.save_for_backward(x, w_gate, w_up, w_down, gate, up)
        ctx.act = act
        if not save:
            return y
        ctx.mark_non_differentiable(gate, up)
        ctx.set_materialize_grads(False)
        return y, gate, up

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, *_):
        return *gated_ff_backward(dy.contiguous(), *ctx.saved_tensors, ctx.act), None, None


# ------------------------------------------------------------------------------------------------ linear layers
def _linear_operands(x, weight, bias, act, gate, rows_per_group):
    """(device, type, type of the parameters, act, rows, width, out_width, row stride of x, of the gate, rows of a group) of checked operands."""
    dev = _current("x", x)
    rows, width, stride = _rows("x", x)
    dtype = x.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        _fail(f"x is {dtype}: bfloat16 and float16 are taken")
    if act not in _LINEAR_ACTS:
        _fail(f"act {act!r} unknown")
    if weight.dim() != 2:
        _fail("weight is a matrix")
    out_width = weight.shape[0]
    if not (weight.dtype is dtype and weight.shape == (out_width, width) and weight.get_device() == dev and weight.is_contiguous()):
        _dense("weight", weight, dev, (out_width, width), dtype)
    kind, gate_stride, group = dtype, out_width, 0
    if bias is not None:
        kind = bias.dtype
        if kind != dtype and kind != _F32:
            _fail(f"bias is {kind}: x's type or float32 is taken")
        _dense("bias", bias, dev, (out_width,), kind)
    if gate is not None:
        group = rows_per_group if rows_per_group > 0 else 0
        gate_kind, gate_stride = _norm_param("gate", gate, dev, dtype, out_width, -(-rows // group) if group else 1)
        if bias is not None and gate_kind != kind:
            _fail("bias and gate differ in their type")
        kind = gate_kind
    return dev, _TYPES[dtype], _TYPES[kind], _LINEAR_ACTS[act], rows, width, out_width, stride, gate_stride, group


@functools.lru_cache(maxsize=256)
def _linear_workspace(dev, shape, backward):
    return hf.hf_linear_workspace(shape, backward)


def linear(x, weight, bias=None, act=None, gate=None, residual=None, rows_per_group=0, save=False):
    """y = residual + gate * act(x weight^T + bias).  x bf16 or f16 [..., width], rows with one common stride; weight [out_width, width] contiguous; bias
    [out_width] of x's type or float32; act None, "silu" or "gelu_tanh"; gate of the bias's types [out_width] or [1, out_width], with rows_per_group
    > 0 [groups, out_width], row r of x taking row r // rows_per_group (slices of a modulation tensor are fine); residual [..., out_width] of x's
    type, rows with one common stride.  save: returns (y, pre), pre = x weight^T + bias [rows, out_width] for `linear_backward`."""
    if _recording() and (x.requires_grad or weight.requires_grad or bias is not None and bias.requires_grad or gate is not None and gate.requires_grad
                         or residual is not None and residual.requires_grad):
        return _Linear.apply(x, weight, bias, act, gate, residual, rows_per_group, save)
    dev, t, pt, a, rows, width, out_width, stride, gate_stride, group = _linear_operands(x, weight, bias, act, gate, rows_per_group)
    residual_stride = out_width
    if residual is not None:
        _like("residual", residual, dev, x.shape[:-1] + (out_width,), x.dtype)
        residual_stride = _rows("residual", residual)[2]
    y = _empty_like(x) if out_width == width == stride else x.new_empty(x.shape[:-1] + (out_width,))
    pre = x.new_empty(rows, out_width) if save else None
    shape = _LINEAR(t, pt, a, width, out_width, rows, stride, out_width, residual_stride, group, gate_stride)
    need = _linear_workspace(dev, shape, 0)
    ws = x.new_empty(need // 2) if need else None
    status = _lib().hf_linear(shape, x.data_ptr(), weight.data_ptr(), bias.data_ptr() if bias is not None else None,
                              gate.data_ptr() if gate is not None else None, residual.data_ptr() if residual is not None else None, y.data_ptr(),
                              pre.data_ptr() if save else None, ws.data_ptr() if need else None, _stream())
    if status:
        _check(status)
    return (y, pre) if save else y


def linear_backward(dy, x, weight, pre=None, act=None, gate=None, rows_per_group=0, dx=True, dweight=True, dbias=True, dgate=True):
    """Gradients of `linear`: (dx, dweight in x's type, dbias float32 [out_width], dgate float32 [groups, out_width]); None for those not asked for (dgate:
    without a gate).  pre: as the forward returned it, needed with an activation or a gate.  The residual's gradient is dy."""
    dev, t, pt, a, rows, width, out_width, stride, gate_stride, group = _linear_operands(x, weight, None, act, gate, rows_per_group)
    _like("dy", dy, dev, x.shape[:-1] + (out_width,), x.dtype)
    if act is not None or gate is not None:
        if pre is None:
            _fail("pre is needed with an activation or a gate")
        _dense("pre", pre, dev, (rows, out_width), x.dtype)
    gx = (_empty_like(x) if stride == width else x.new_empty(x.shape)) if dx else None
    gw = _empty_like(weight) if dweight else None
    gb = _empty_strided((out_width,), (1,), dtype=_F32, device=x.device) if dbias else None
    gg = _empty_strided((-(-rows // group) if group else 1, out_width), (out_width, 1), dtype=_F32, device=x.device) if dgate and gate is not None else None
    shape = _LINEAR(t, pt, a, width, out_width, rows, stride, _rows("dy", dy)[2], out_width, group, gate_stride)
    ws = x.new_empty(_linear_workspace(dev, shape, 1) // 2)
    status = _lib().hf_linear_backward(shape, dy.data_ptr(), x.data_ptr(), weight.data_ptr(), pre.data_ptr() if pre is not None else None,
                                       gate.data_ptr() if gate is not None else None, gx.data_ptr() if dx else None, gw.data_ptr() if dweight else None,
                                       gb.data_ptr() if dbias else None, gg.data_ptr() if gg is not None else None, ws.data_ptr(), _stream())
    if status:
        _check(status)
    return gx, gw, gb, gg


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, gate, residual, rows_per_group, save):
        kept = act is not None or gate is not None
        y, pre = linear(x, weight, bias, act, gate, residual, rows_per_group, True) if save or kept else (linear(x, weight, bias, None, None, residual), None)
        ctx.save_for_backward(x, weight, gate, pre if kept else None)
        ctx.args, ctx.bias = (act, rows_per_group), None if bias is None else bias.dtype
        if not save:
            return y
        ctx.mark_non_differentiable(pre)
        ctx.set_materialize_grads(False)
        return y, pre

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, *_):
        x, weight, gate, pre = ctx.saved_tensors
        act, group = ctx.args
        need = ctx.needs_input_grad
        dy = dy.contiguous()
        dx, dw, db, dg = linear_backward(dy, x, weight, pre, act, gate, group, need[0], need[1], need[2], need[4])
        return (dx, dw, db.to(ctx.bias) if need[2] else None, None, dg.view(gate.shape).to(gate.dtype) if need[4] else None, dy if need[5] else None, None, None)
