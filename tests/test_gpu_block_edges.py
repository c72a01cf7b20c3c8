"""The denoiser block where it can go wrong without an error: types, selections made in between, chunks that follow one another."""
import pytest
import torch

pytestmark = pytest.mark.gpu
HIGH, WIDE = 8, 12


def build(keep=500, batch=1, window=2, **kw):
    from paper_2604_10103_b200 import binding as hf, block as bl, inputs as gen
    w = gen.Workload("edges", batch=batch, heads=3, head_dim=64, tokens_per_frame=HIGH * WIDE, chunk_frames=4, window_frames=4 * window,
                     block=128, topk=0, keep_permille=keep, seed=3)
    ctx = hf.Context(hf.make_config(w, merge=hf.HF_MERGE_IDENTITY))
    torch.manual_seed(5)
    return w, ctx, bl.DenoiserBlock(w, HIGH, WIDE, ctx, **kw)


def chunk(w, seed):
    g = torch.Generator().manual_seed(seed)
    width = w.heads * w.head_dim
    return (torch.randn(w.batch, w.chunk_tokens, width, generator=g).bfloat16().cuda(),
            (0.3 * torch.randn(w.batch, w.chunk_frames, 6, width, generator=g)).bfloat16().cuda())


def test_autocast_to_another_type_is_refused():
    w, ctx, b = build()
    x, mod = chunk(w, 1)
    ref = b(x, mod, b.positions(0))
    for call in (b.forward, b.commit):
        with torch.autocast("cuda", dtype=torch.float16), pytest.raises(ValueError, match="projection is torch.float16"):
            call(x, mod, b.positions(0))
    with torch.autocast("cuda", dtype=torch.bfloat16):
        assert torch.equal(b(x, mod, b.positions(0)), ref)


def gradients(b, xs, mods, between=None, order=None):
    """The chunks' gradients, all forward passes before the first backward pass."""
    xs, ys = [x.clone().requires_grad_() for x in xs], []
    b.zero_grad(set_to_none=True)
    for x, mod in zip(xs, mods):
        ys.append(b(x, mod, b.positions(4)))
    if between:
        between()
    for i in order or range(len(xs)):
        ys[i].float().square().sum().backward()
    return [x.grad for x in xs] + [p.grad for p in b.parameters()]


def test_forward_passes_of_one_layer_before_the_first_backward_pass():
    """Each gradient is that of its own selection, whichever was made last."""
    w, ctx, b = build()
    with torch.no_grad():
        x, mod = chunk(w, 0)
        b.commit(x, mod, b.positions(0))
    (x1, m1), (x2, m2) = chunk(w, 1), chunk(w, 2)
    alone = [gradients(b, [x], [m]) for x, m in ((x1, m1), (x2, m2))]
    both = gradients(b, [x1, x2], [m1, m2])
    assert torch.equal(both[0], alone[0][0]) and torch.equal(both[1], alone[1][0])
    back = gradients(b, [x1, x2], [m1, m2], order=[1, 0])
    assert torch.equal(back[0], alone[0][0]) and torch.equal(back[1], alone[1][0])

    def another():
        with torch.no_grad():
            b(x2, m2, b.positions(4))
    assert all(torch.equal(p, q) for p, q in zip(gradients(b, [x1], [m1], another), alone[0]))


def test_a_cache_or_state_that_has_changed_before_the_backward_pass():
    w, ctx, b = build()
    x, mod = chunk(w, 1)
    k = torch.randn(w.batch, w.heads, 64, w.head_dim, device="cuda").bfloat16()

    def commit():
        with torch.no_grad():
            b.commit(x, mod, b.positions(0))
    for between in (commit, lambda: ctx.hf_state_absorb(0, k, k, 64), lambda: ctx.hf_reset(0), lambda: ctx.hf_reset(),
                    lambda: ctx.hf_state_import(ctx.hf_state_export())):
        with pytest.raises(RuntimeError, match="has changed since the forward pass"):
            gradients(b, [x], [mod], between)
    gradients(b, [x], [mod])


def test_second_derivatives_are_refused():
    w, ctx, b = build()
    x, mod = chunk(w, 1)
    x.requires_grad_()
    g, = torch.autograd.grad(b(x, mod, b.positions(0)).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.float().square().sum().backward()


def test_the_attention_alone_refuses_a_second_derivative():
    from paper_2604_10103_b200 import block as bl
    w, ctx, b = build()
    q, k, v = (torch.randn(w.batch, w.heads, w.chunk_tokens, w.head_dim, device="cuda").bfloat16().requires_grad_() for _ in range(3))
    g, = torch.autograd.grad(bl._Attention.apply(q, k, v, ctx, 0).float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.float().square().sum().backward()


def test_positions_that_change_before_the_backward_pass_are_seen():
    w, ctx, b = build()
    x, mod = chunk(w, 1)
    pos = b.positions(0)
    y = b(x.requires_grad_(), mod, pos)
    pos += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()


def test_time_from_the_context():
    """The relative temporal rotation of the library in place of the time axis: the same angles between queries and keys, so the same attention (all
    blocks kept, nothing in the history).  q and k are rounded once more on the way (U each, and the keys of the cache); the rest is the same."""
    import numpy as np
    from tests import layer_forms as lf

    def stream(own):
        w, ctx, b = build(keep=1000, window=3)
        if not own:
            n, t0 = b.pairs[0], 40
            th = np.arange(t0 + 1)[:, None] * 10000.0 ** (-np.arange(n) / n)[None, :]
            ctx.hf_set_temporal_rope(t0, 0, n, torch.from_numpy(np.cos(th).astype(np.float32)).cuda(), torch.from_numpy(np.sin(th).astype(np.float32)).cuda())
        out = []
        with torch.no_grad():
            for i in range(3):
                x, mod = chunk(w, i)
                pos = b.positions(i * w.chunk_frames)
                if not own:
                    pos[:, 0] = 0
                out.append(b(x, mod, pos))
                b.commit(x, mod, pos)
        assert ctx.hf_get_device_status() == (0, 0)
        return out
    for got, ref in zip(stream(False), stream(True)):
        assert lf.rel(got, lf.f64(ref)) < 3 * lf.U[torch.bfloat16]
