"""A denoiser block around the hybrid attention: modulated layer norm, fused projection, rotary positions in time, height and width, hybrid
attention, output projection; modulated layer norm, gated feed-forward; a gated residual after each half.

`DenoiserBlock.forward` is one layer of one denoising step of a stream (no gradient), `commit` folds a finished chunk into the layer's cache and
state, and `forward` under autograd is the step with gradient: every operator between the projections has its backward pass in the
library, and the plain projections are torch's.  `python -m paper_2604_10103_b200.block` runs a short stream and one training step at the
832x480 shape on synthetic data and prints their times.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as hf
from . import inputs as gen
from . import layers
from . import rope


class _Attention(torch.autograd.Function):
    """The hybrid attention of one layer for the step with gradient: its selection is held fixed, the cached chunks and the state get no
    gradient (Alg. 1).  The context must keep this layer's cache and state until the backward pass, which refuses others; a selection that
    has replaced this one's in between is made anew (the same q, k and cache: the same selection)."""

    @staticmethod
    def forward(ctx, q, k, v, context, layer):
        o, o_hist = torch.empty_like(q), torch.empty_like(q)
        lse = q.new_empty(q.shape[:3], dtype=torch.float32)
        context.hf_block_select(layer, q, k)
        context.hf_sparse_swa(layer, q, k, v, o, lse=lse)
        context.hf_linear_attn(layer, q, o_hist)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.context, ctx.layer, ctx.selection, ctx.change = context, layer, context.selections[layer], context.changes[layer]
        return o + o_hist

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        q, k, v, o, lse = ctx.saved_tensors
        context, layer = ctx.context, ctx.layer
        if context.changes[layer] != ctx.change:
            raise RuntimeError(f"the cache or state of layer {layer} has changed since the forward pass")
        if context.selections[layer] != ctx.selection:
            context.hf_block_select(layer, q, k)
            ctx.selection = context.selections[layer]
        g = g.contiguous()
        dq, dq_hist, dk, dv = (torch.empty_like(q) for _ in range(4))
        context.hf_sparse_swa_backward_dq(layer, q, k, v, o, lse, g, dq)
        context.hf_sparse_swa_backward_dkv(layer, q, k, v, o, lse, g, dk, dv)
        context.hf_linear_attn_backward_dq(layer, q, g, dq_hist)
        return dq + dq_hist, dk, dv, None, None


def _bf16(name, t):
    """The attention takes bare pointers: a type that it would misread is refused here."""
    if t.dtype is not torch.bfloat16:
        raise ValueError(f"{name} is {t.dtype}: the hybrid attention takes bfloat16")


class DenoiserBlock(torch.nn.Module):
    """One layer.  w: an `inputs.Workload` (batch, heads, head_dim, frames); high x wide tokens a frame; context: the `binding.Context`
    that holds the layer's cache and state; last_frame: the last frame of the stream in the time table (8 bytes a frame and pair: a million
    frames of a head of 128 take 176 MB).  A stream without an end has its time from the context: with `hf_set_temporal_rope` for the pairs
    0 .. pairs[0] - 1 the library turns and re-indexes them, and the positions given here are 0 on the time axis (no gradient then)."""

    def __init__(self, w, high, wide, context, layer=0, hidden=None, act="silu", last_frame=255, eps=1e-6, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        if high * wide != w.tokens_per_frame:
            raise ValueError(f"{high} x {wide} tokens are not a frame of {w.tokens_per_frame}")
        if dtype is not torch.bfloat16:
            raise ValueError(f"the weights are {dtype}: the hybrid attention takes bfloat16")
        c = context.cfg
        if (c.batch, c.heads, c.head_dim, c.tokens_per_frame * c.chunk_frames) != (w.batch, w.heads, w.head_dim, w.chunk_tokens):
            raise ValueError("the context's batch, heads, head_dim or tokens of a chunk are not the workload's")
        self.w, self.context, self.layer, self.act, self.eps = w, context, layer, act, eps
        width = w.heads * w.head_dim
        hidden = hidden or (8 * width // 3 + 63) // 64 * 64

        def matrix(n_out, n_in):
            return torch.nn.Parameter(torch.randn(n_out, n_in, device=device).mul_(n_in ** -0.5).to(dtype))
        self.w_qkv, self.w_out = matrix(3 * width, width), matrix(width, width)
        self.w_gate, self.w_up, self.w_down = matrix(hidden, width), matrix(hidden, width), matrix(width, hidden)
        n = w.head_dim // 2
        self.pairs, self.extents = (n - 2 * (n // 3), n // 3, n // 3), (last_frame + 1, high, wide)
        cos, sin = rope.axis_tables(self.extents, self.pairs)
        self.register_buffer("cos", torch.from_numpy(cos).to(device))
        self.register_buffer("sin", torch.from_numpy(sin).to(device))
        grid = torch.meshgrid(torch.arange(w.chunk_frames), torch.arange(high), torch.arange(wide), indexing="ij")
        self.register_buffer("pos", torch.stack([g.reshape(-1) for g in grid], dim=1).to(torch.int32).to(device))

    def positions(self, first_frame):
        """Positions of the chunk whose first frame is the stream's frame `first_frame` (from 0)."""
        if not 0 <= first_frame <= self.extents[0] - self.w.chunk_frames:
            raise ValueError(f"frames {first_frame} .. {first_frame + self.w.chunk_frames - 1} are not in the time table: last_frame is {self.extents[0] - 1}")
        pos = self.pos.clone()
        pos[:, 0] += first_frame
        return pos

    def _norm(self, x, scale, shift):
        """xhat (1 + scale) + shift, one row of scale and shift [batch, frames, width] for the tokens of a frame."""
        width = x.shape[-1]
        return layers.layer_norm(x, scale.reshape(-1, width), shift.reshape(-1, width), eps=self.eps, weight_offset=1.0,
                                 rows_per_group=self.w.tokens_per_frame)[0]

    def _heads(self, x, mod, pos):
        taken = [self.w.batch, self.w.chunk_tokens, self.w.heads * self.w.head_dim]
        if list(x.shape) != taken:              # (the attention reads and writes as much, whatever it is given)
            raise ValueError(f"x is {list(x.shape)}: {taken} is taken")
        _bf16("x", x)
        if x.get_device() != self.context.device:
            raise ValueError(f"x is on {x.device}, the context on device {self.context.device}")
        h = self._norm(x, mod[:, :, 1], mod[:, :, 0])
        qkv = torch.nn.functional.linear(h, self.w_qkv)
        _bf16("the projection", qkv)            # (autocast may have changed its type)
        return layers.split_heads_rope(qkv, self.w.heads, self.w.heads, pos, (self.cos, self.sin, self.extents, self.pairs))

    def forward(self, x, mod, pos):
        """x [batch, tokens of a chunk, width]; mod [batch, frames of the chunk, 6, width]: shift, scale, gate of the attention half, then of the
        feed-forward's; pos: `positions` of the chunk's first frame."""
        q, k, v = self._heads(x, mod, pos)
        if torch.is_grad_enabled() and q.requires_grad:
            o = _Attention.apply(q, k, v, self.context, self.layer)
        else:
            o = torch.empty_like(q)
            self.context.hf_hybrid_forward(self.layer, q, k, v, o)
        per_token = mod.repeat_interleave(self.w.tokens_per_frame, dim=1)
        x = x + per_token[:, :, 2] * torch.nn.functional.linear(o.transpose(1, 2).flatten(2), self.w_out)
        h = self._norm(x, mod[:, :, 4], mod[:, :, 3])
        y = layers.gated_ff(h, self.w_gate, self.w_up, self.w_down, act=self.act)
        return x + per_token[:, :, 5] * y

    @torch.no_grad()
    def commit(self, x, mod, pos):
        """The finished chunk's keys and values go into the layer's cache (and the oldest chunk into its state)."""
        _, k, v = self._heads(x, mod, pos)
        self.context.hf_kv_append(self.layer, k, v)


def main():
    w = gen.layer_832x480()
    context = hf.Context(hf.make_config(w, merge=hf.HF_MERGE_IDENTITY))
    torch.manual_seed(0)
    block = DenoiserBlock(w, 30, 52, context)
    T, width = w.chunk_frames * w.tokens_per_frame, w.heads * w.head_dim

    def chunk():
        return torch.randn(w.batch, T, width, device="cuda").bfloat16(), 0.3 * torch.randn(w.batch, w.chunk_frames, 6, width, device="cuda").bfloat16()

    def timed(f):
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        for _ in range(3):
            f()
        e[0].record()
        for _ in range(10):
            f()
        e[1].record()
        torch.cuda.synchronize()
        return e[0].elapsed_time(e[1]) / 10

    with torch.no_grad():
        for i in range(4):
            x, mod = chunk()
            y = block(x, mod, block.positions(i * w.chunk_frames))
            block.commit(y, mod, block.positions(i * w.chunk_frames))
        x, mod = chunk()
        pos = block.positions(4 * w.chunk_frames)
        print(f"one layer of one denoising step, {T} tokens: {timed(lambda: block(x, mod, pos)):.3f} ms")
    x.requires_grad_()

    def step():
        block.zero_grad(set_to_none=True)
        block(x, mod, pos).float().square().mean().backward()
    print(f"the same with gradient: {timed(step):.3f} ms")
    context.hf_get_device_status()
    hf.hf_layers_status()


if __name__ == "__main__":
    main()
