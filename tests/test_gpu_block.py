"""The denoiser block: its operators together with the hybrid attention, against a 64-bit model in which the attention is dense (all blocks kept,
nothing in the history), forward and gradients; and as a stream."""
import numpy as np
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
HIGH, WIDE = 8, 12


def build(dtype=torch.bfloat16, keep=1000, window=2, batch=1, act="silu"):
    from paper_2604_10103_b200 import binding as hf, block as bl, inputs as gen
    w = gen.Workload("block", batch=batch, heads=3, head_dim=64, tokens_per_frame=HIGH * WIDE, chunk_frames=2, window_frames=2 * window,
                     block=128, topk=0, keep_permille=keep, seed=3)
    ctx = hf.Context(hf.make_config(w, merge=hf.HF_MERGE_IDENTITY))
    torch.manual_seed(5)
    return w, ctx, bl.DenoiserBlock(w, HIGH, WIDE, ctx, act=act)


def reference(b, x, mod, pos, params):
    """The block in 64 bits on the CPU with dense attention; params: dict of 64-bit matrices."""
    w, frame = b.w, b.w.tokens_per_frame

    def norm(v, shift, scale):
        m = v.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt((v - m).square().mean(-1, keepdim=True) + b.eps)
        return (v - m) * r * (1.0 + scale.repeat_interleave(frame, 1)) + shift.repeat_interleave(frame, 1)

    B, T, width = x.shape
    cos, sin, at, start = b.cos.double().cpu(), b.sin.double().cpu(), [], 0
    for a, (e, n) in enumerate(zip(b.extents, b.pairs)):
        at.append(start + pos[:, a:a + 1].cpu().long() * n + torch.arange(n))
        start += e * n
    at = torch.cat(at, dim=1)
    c, s = cos[at][:, None], sin[at][:, None]

    def turn(v):
        x0, x1 = v[..., 0::2], v[..., 1::2]
        return torch.stack([x0 * c - x1 * s, x0 * s + x1 * c], dim=-1).flatten(-2)

    h = norm(x, mod[:, :, 0], mod[:, :, 1])
    q, k, v = (h @ params["w_qkv"].t()).view(B, T, 3, w.heads, w.head_dim).unbind(2)
    q, k = turn(q), turn(k)
    p = torch.softmax(torch.einsum("bthd,bshd->bhts", q, k) * w.head_dim ** -0.5, dim=-1)
    o = torch.einsum("bhts,bshd->bthd", p, v).flatten(2)
    x = x + mod[:, :, 2].repeat_interleave(frame, 1) * (o @ params["w_out"].t())
    h = norm(x, mod[:, :, 3], mod[:, :, 4])
    y = (lf.act(h @ params["w_gate"].t(), b.act) * (h @ params["w_up"].t())) @ params["w_down"].t()
    return x + mod[:, :, 5].repeat_interleave(frame, 1) * y


NAMES = ("w_qkv", "w_out", "w_gate", "w_up", "w_down")


@pytest.mark.parametrize("batch,act", [(1, "silu"), (2, "gelu_tanh")])
def test_forward_and_gradients_against_a_dense_model(batch, act):
    """About ten roundings to bf16 follow one another (norm, projection, rotation, p, o, projection, residual, ...), each of at most U in the
    2-norm and independent: sqrt(10) U forward; a gradient passes through both directions and the rounded saved tensors: twice that."""
    w, ctx, b = build(batch=batch, act=act)
    width, T = w.heads * w.head_dim, w.chunk_frames * w.tokens_per_frame
    g = torch.Generator().manual_seed(1)
    x = torch.randn(batch, T, width, generator=g).bfloat16()
    mod = (0.3 * torch.randn(batch, w.chunk_frames, 6, width, generator=g)).bfloat16()
    dy = torch.randn(batch, T, width, generator=g).bfloat16()
    pos = b.positions(7)
    xg, mg = x.cuda().requires_grad_(), mod.cuda().requires_grad_()
    y = b(xg, mg, pos)
    y.backward(dy.cuda())
    x64, m64 = x.double().requires_grad_(), mod.double().requires_grad_()
    params = {n: lf.f64(getattr(b, n)).requires_grad_() for n in NAMES}
    ref = reference(b, x64, m64, pos, params)
    ref.backward(dy.double())
    u = lf.U[torch.bfloat16]
    assert lf.rel(y, ref.detach()) < 10 ** 0.5 * u
    for name, got, want in [("x", xg.grad, x64.grad), ("mod", mg.grad, m64.grad)] + [(n, getattr(b, n).grad, params[n].grad) for n in NAMES]:
        assert lf.rel(got, want) < 2 * 10 ** 0.5 * u, name
    with torch.no_grad():
        assert lf.rel(b(x.cuda(), mod.cuda(), pos), ref.detach()) < 10 ** 0.5 * u
    from paper_2604_10103_b200 import binding as hf
    assert ctx.hf_get_device_status() == (0, 0) and hf.hf_layers_status() == (0, 0)


def test_a_stream_of_chunks():
    """Four chunks through the block: positions run on, the window fills, the oldest chunk leaves into the state; repeated, the same bits."""
    def run():
        w, ctx, b = build(keep=500, window=2)
        width, T = w.heads * w.head_dim, w.chunk_frames * w.tokens_per_frame
        g = torch.Generator().manual_seed(2)
        out = []
        with torch.no_grad():
            for i in range(4):
                x = torch.randn(1, T, width, generator=g).bfloat16().cuda()
                mod = (0.3 * torch.randn(1, w.chunk_frames, 6, width, generator=g)).bfloat16().cuda()
                pos = b.positions(i * w.chunk_frames)
                for _ in range(2):
                    x = b(x, mod, pos)
                b.commit(x, mod, pos)
                out.append(x.clone())
        from paper_2604_10103_b200 import binding as hf
        assert ctx.hf_query(0, hf.HF_Q_ABSORBED_TOKENS) == 3 * T
        assert ctx.hf_get_device_status() == (0, 0) and hf.hf_layers_status() == (0, 0)
        return out
    first, second = run(), run()
    assert all(torch.isfinite(a).all() and torch.equal(a, c) for a, c in zip(first, second))
