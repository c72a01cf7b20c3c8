"""The block with biases, norms of q and k and a feed-forward of two matrices: against a 64-bit model with dense attention (all blocks kept, nothing in the
history), forward and gradients; as a stream; and a training step with the gradients' norm and AdamW."""
import math

import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
HIGH, WIDE = 8, 12
NAMES = ("w_qkv", "b_qkv", "q_norm", "k_norm", "w_out", "b_out", "w_first", "b_first", "w_second", "b_second")


def build(norm_over="width", batch=1, keep=1000, window=2, act="gelu_tanh"):
    from paper_2604_10103_b200 import binding as hf, block as bl, inputs as gen
    w = gen.Workload("biased", batch=batch, heads=3, head_dim=64, tokens_per_frame=HIGH * WIDE, chunk_frames=2, window_frames=2 * window,
                     block=128, topk=0, keep_permille=keep, seed=3)
    ctx = hf.Context(hf.make_config(w, merge=hf.HF_MERGE_IDENTITY))
    torch.manual_seed(5)
    b = bl.BiasedBlock(w, HIGH, WIDE, ctx, act=act, norm_over=norm_over)
    with torch.no_grad():
        for n in NAMES:
            if n[:2] == "b_" or n[2:] == "norm":
                getattr(b, n).add_(0.3 * torch.randn_like(getattr(b, n)))
    return w, ctx, b


def chunk(w, seed=1):
    g = torch.Generator().manual_seed(seed)
    width, T = w.heads * w.head_dim, w.chunk_frames * w.tokens_per_frame
    return (torch.randn(w.batch, T, width, generator=g).bfloat16(), (0.3 * torch.randn(w.batch, w.chunk_frames, 6, width, generator=g)).bfloat16(),
            torch.randn(w.batch, T, width, generator=g).bfloat16())


def reference(b, x, mod, pos, p):
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

    def turned(v, weight):
        over = (-2, -1) if weight.numel() == width else (-1,)
        v = v / torch.sqrt(v.square().mean(over, keepdim=True) + b.eps) * weight.view(-1, w.head_dim)
        x0, x1 = v[..., 0::2], v[..., 1::2]
        return torch.stack([x0 * c - x1 * s, x0 * s + x1 * c], dim=-1).flatten(-2)
    h = norm(x, mod[:, :, 0], mod[:, :, 1])
    q, k, v = (h @ p["w_qkv"].t() + p["b_qkv"]).view(B, T, 3, w.heads, w.head_dim).unbind(2)
    a = torch.softmax(torch.einsum("bthd,bshd->bhts", turned(q, p["q_norm"]), turned(k, p["k_norm"])) * w.head_dim ** -0.5, dim=-1)
    o = torch.einsum("bhts,bshd->bthd", a, v).flatten(2)
    x = x + mod[:, :, 2].repeat_interleave(frame, 1) * (o @ p["w_out"].t() + p["b_out"])
    h = lf.act(norm(x, mod[:, :, 3], mod[:, :, 4]) @ p["w_first"].t() + p["b_first"], b.act)
    return x + mod[:, :, 5].repeat_interleave(frame, 1) * (h @ p["w_second"].t() + p["b_second"])


@pytest.mark.parametrize("norm_over,batch,act", [("width", 1, "gelu_tanh"), ("head", 2, "silu")])
def test_forward_and_gradients_against_a_dense_model(norm_over, batch, act):
    """About ten roundings to bf16 follow one another (norm, projection, rotation, p, o, projection, hidden, ...), each of at most U in the 2-norm and
    independent: sqrt(10) U forward; a gradient passes through both directions and the rounded saved tensors: twice that."""
    w, ctx, b = build(norm_over, batch, act=act)
    x, mod, dy = chunk(w)
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


def test_a_stream_repeats_its_bits():
    from paper_2604_10103_b200 import binding as hf

    def run():
        w, ctx, b = build(keep=500)
        out = []
        with torch.no_grad():
            for i in range(5):
                x, mod, _ = (t.cuda() for t in chunk(w, seed=i))
                y = b(x, mod, b.positions(2 * i))
                b.commit(y, mod, b.positions(2 * i))
                out.append(y)
        assert ctx.hf_get_device_status() == (0, 0) and hf.hf_layers_status() == (0, 0)
        return out
    first, second = run(), run()
    assert all(torch.isfinite(a).all() and torch.equal(a, c) for a, c in zip(first, second))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step(bits):
    """Backward, the norm of all gradients, a step of AdamW: the masters move as the definition says for the gradients that the backward pass gave.  A first
    step's quotient is +-1 (up to eps), so each element moves by lr, apart from the decay, within float32 (see the optimizer's own tests)."""
    from paper_2604_10103_b200 import optim
    w, ctx, b = build()
    opt = optim.AdamW(b.parameters(), lr=1e-2, eps=1e-12, weight_decay=0.1, state_bits=bits)
    x, mod, dy = (t.cuda() for t in chunk(w))
    for step in range(2):
        opt.zero_grad()
        b(x, mod, b.positions(0)).backward(dy)
        params = list(b.parameters())
        norm, factor = optim.gradient_norm([p.grad for p in params], max_norm=0.5)
        want = math.sqrt(sum(float(lf.f64(p.grad).square().sum()) for p in params))
        assert abs(float(norm) - want) <= 1e-5 * want and abs(float(factor) - min(1.0, 0.5 / want)) <= 1e-5
        before = [lf.f64(opt.state[p]["master"]) for p in params]
        grads = [lf.f64(p.grad) for p in params]
        opt.step(grad_factor=factor)
        for p, old, g in zip(params, before, grads):
            master = opt.state[p]["master"]
            assert torch.equal(p.detach(), master.bfloat16()) and torch.isfinite(p).all()
            if step == 0:
                moved = lf.f64(master) - old * (1 - 1e-3)
                large = g.abs() * float(factor) > 1e-8          # (eps does not show)
                assert ((moved + 1e-2 * torch.sign(g)).abs() <= 1e-2 * 1e-3 + 1e-6 * old.abs())[large].all()


def test_the_command_trains(capsys):
    from paper_2604_10103_b200 import block as bl
    bl.main()
    out = capsys.readouterr().out
    assert out.count(" ms") == 5 and "AdamW" in out
