"""The operators of `layers` on tensors that need gradients: they are part of torch's graph."""
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def leaf(*shape, seed=0, dtype=BF, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda().requires_grad_()


def grads(out, inputs, dout, **kw):
    return torch.autograd.grad(out, inputs, dout, **kw)


@pytest.mark.parametrize("group,offset", [(0, 0.0), (0, 1.0), (7, 1.0)])
@pytest.mark.parametrize("param", [BF, F32])
def test_layer_norm(group, offset, param):
    from paper_2604_10103_b200 import layers
    rows, width = 21, 96
    groups = 3 if group else 1
    x, w, b = leaf(rows, width), leaf(groups, width, seed=1, dtype=param), leaf(groups, width, seed=2, dtype=param)
    dy = leaf(rows, width, seed=3).detach()
    y, mean, rstd = layers.layer_norm(x, w, b, weight_offset=offset, rows_per_group=group)
    assert y.requires_grad and not mean.requires_grad and not rstd.requires_grad
    with torch.no_grad():
        y0, mean0, rstd0 = layers.layer_norm(x, w, b, weight_offset=offset, rows_per_group=group)
        want = layers.layer_norm_backward(dy, x, mean0, rstd0, w, weight_offset=offset, rows_per_group=group)
    assert not y0.requires_grad and torch.equal(y, y0) and torch.equal(mean, mean0) and torch.equal(rstd, rstd0)
    dx, dw, db = grads(y, (x, w, b), dy)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1].to(param)) and torch.equal(db, want[2].to(param))
    # gradients that are broadcast or lie across: as their copies
    y = layers.layer_norm(x, w, b, weight_offset=offset, rows_per_group=group)[0]
    one = torch.ones((), dtype=BF, device="cuda")
    assert all(torch.equal(p, q) for p, q in zip(grads(y, (x, w, b), one.expand(rows, width), retain_graph=True), grads(y, (x, w, b), torch.ones_like(y), retain_graph=True)))
    assert torch.equal(grads(y, (x,), dy.t().contiguous().t())[0], dx)


def test_layer_norm_with_some_inputs():
    from paper_2604_10103_b200 import layers
    x, w, b = leaf(2, 5, 64), leaf(64, seed=1), leaf(64, seed=2)
    dy = leaf(2, 5, 64, seed=3).detach()
    dx, dw, db = grads(layers.layer_norm(x, w, b)[0], (x, w, b), dy)
    assert dx.shape == x.shape and dw.shape == w.shape == db.shape
    assert torch.equal(grads(layers.layer_norm(x.detach(), w, b)[0], (w,), dy)[0], dw)
    assert torch.equal(grads(layers.layer_norm(x.detach(), None, b)[0], (b,), dy)[0], db)
    assert torch.equal(grads(layers.layer_norm(x, w.detach(), b.detach())[0], (x,), dy)[0], dx)
    y, mean, _ = layers.layer_norm(x)
    dx = grads(y, (x,), dy)[0]
    assert torch.equal(dx, layers.layer_norm_backward(dy, x.detach(), mean, layers.layer_norm(x.detach())[2])[0])


def tables():
    from paper_2604_10103_b200 import rope
    extents, pairs = (6, 5, 4), (12, 10, 10)
    cos, sin = rope.axis_tables(extents, pairs)
    g = torch.Generator().manual_seed(4)
    pos = torch.stack([torch.randint(0, e, (33,), generator=g) for e in extents], dim=1).to(torch.int32).cuda()
    return (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), extents, pairs), pos


def test_rotary_positions():
    from paper_2604_10103_b200 import layers
    tab, pos = tables()
    for inverse in (False, True):
        x, dy = leaf(2, 33, 3, 64), leaf(2, 33, 3, 64, seed=1).detach()
        y = layers.rope_axes(x, pos, tab, inverse=inverse)
        assert torch.equal(y, layers.rope_axes(x.detach(), pos, tab, inverse=inverse))
        want = layers.rope_axes(dy, pos, tab, inverse=not inverse)
        assert torch.equal(grads(y, (x,), dy, retain_graph=True)[0], want)
        across = torch.empty(64, 2, 33, 3, dtype=BF, device="cuda").permute(1, 2, 3, 0).copy_(dy)
        assert across.stride(-1) != 1 and torch.equal(grads(y, (x,), across)[0], want)
        out = torch.empty_like(x)
        with pytest.raises(ValueError, match="out"):
            layers.rope_axes(x, pos, tab, out=out.detach())
        with torch.no_grad():
            layers.rope_axes(x, pos, tab, out=out)


@pytest.mark.parametrize("H,KV,pairing", [(4, 4, "adjacent"), (4, 2, "adjacent"), (4, 1, "halves")])
def test_fused_projection(H, KV, pairing):
    from paper_2604_10103_b200 import layers
    tab, pos = tables()
    x = leaf(2, 33, (H + 2 * KV) * 64)
    q, k, v = layers.split_heads_rope(x, H, KV, pos, tab, pairing=pairing)
    dq, dk, dv = (leaf(*t.shape, seed=i).detach() for i, t in enumerate((q, k, v)))
    want = layers.split_heads_rope_backward(dq, dk, dv, pos, tab, pairing=pairing)
    assert torch.equal(grads((q, k, v), (x,), (dq, dk, dv), retain_graph=True)[0], want)
    zero = [torch.zeros_like(t) for t in (dq, dk, dv)]
    # the sum's gradient is one number for all elements; k takes no part
    got = torch.autograd.grad(q.sum() + v.sum(), x, retain_graph=True)[0]
    assert torch.equal(got, layers.split_heads_rope_backward(torch.ones_like(q), zero[1], torch.ones_like(v), pos, tab, pairing=pairing))
    across = torch.empty(64, *q.shape[:3], dtype=BF, device="cuda").permute(1, 2, 3, 0).copy_(dq)
    assert torch.equal(grads((q, k, v), (x,), (across, dk, dv))[0], want)


@pytest.mark.parametrize("M", [5, 60])
def test_feed_forward(M):
    from paper_2604_10103_b200 import layers
    K, N, O = 64, 136, 72
    x, wg, wu, wd = leaf(M, K), leaf(N, K, seed=1, scale=K ** -0.5), leaf(N, K, seed=2, scale=K ** -0.5), leaf(O, N, seed=3, scale=N ** -0.5)
    dy = leaf(M, O, seed=4).detach()
    for act in ("silu", "gelu_tanh"):
        with torch.no_grad():
            y0, gate, up = layers.gated_ff(x, wg, wu, wd, act=act, save=True)
            want = layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up, act=act)
        for save in (False, True):
            out = layers.gated_ff(x, wg, wu, wd, act=act, save=save)
            y = out[0] if save else out
            assert torch.equal(y, y0) and (not save or not (out[1].requires_grad or out[2].requires_grad))
            assert all(torch.equal(p, q) for p, q in zip(grads(y, (x, wg, wu, wd), dy, retain_graph=True), want))
            assert torch.equal(grads(y, (x,), torch.ones((), dtype=BF, device="cuda").expand(M, O), retain_graph=True)[0], grads(y, (x,), torch.ones_like(y))[0])
        assert torch.equal(grads(layers.gated_ff(x, wg.detach(), wu.detach(), wd.detach(), act=act), (x,), dy)[0], want[0])
        assert torch.equal(grads(layers.gated_ff(x.detach(), wg, wu.detach(), wd.detach(), act=act), (wg,), dy)[0], want[1])


def test_what_changes_between_the_passes_is_seen():
    from paper_2604_10103_b200 import layers
    tab, pos = tables()
    x = leaf(1, 33, 6 * 64)
    for moved in (pos, tab[0], tab[1]):
        q, k, v = layers.split_heads_rope(x, 2, 2, pos, tab)
        moved.add_(0)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            q.sum().backward()


def test_second_derivatives_are_refused():
    from paper_2604_10103_b200 import layers
    tab, pos = tables()
    x, w = leaf(1, 33, 6 * 64), leaf(6 * 64, seed=1)
    wg, wd = leaf(64, 6 * 64, seed=2), leaf(64, 64, seed=3)
    for f in (lambda: layers.layer_norm(x, w)[0], lambda: layers.split_heads_rope(x, 2, 2, pos, tab)[0], lambda: layers.gated_ff(x, wg, wg, wd),
              lambda: layers.rope_axes(x.view(1, 33, 6, 64), pos, tab)):
        g, = torch.autograd.grad(f().float().square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.float().square().sum().backward()
