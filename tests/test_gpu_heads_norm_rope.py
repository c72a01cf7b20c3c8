"""Norms of q and k with the rotation and the split into heads, against the definition in 64 bits.

Bounds.  The mean of n squares carries a float32 sum's error, at most n 2^-24 of itself, r half of that and four roundings; q two products and a
rotation (4 2^-24 of |x0| + |x1|), then one rounding: U |q| + (n / 2 + 16) 2^-24 (|x0| + |x1|) r w.  The backward pass adds the mean of n products:
(n + 16) 2^-24 of their absolute terms.  The weights' gradients are float32 sums of N terms: (N + n + 32) 2^-24 of the absolute ones."""
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32
E = 2.0 ** -24


@pytest.fixture(autouse=True)
def no_position_outside():
    yield
    from paper_2604_10103_b200 import binding as hf
    assert hf.hf_layers_status() == (0, 0)


def make(B, T, H, KV, d, dtype, over, extents, pairs, seed=0, wtype=None):
    g = torch.Generator().manual_seed(seed + T * 7 + H * 31 + d)
    size = torch.exp(torch.randn(H + 2 * KV, 1, generator=g)).expand(-1, d).reshape(-1)
    qkv = (torch.randn(B, T, (H + 2 * KV) * d, generator=g) * size).to(dtype).cuda()
    n = (1, 1) if over == "head" else (H, KV)
    qw, kw = ((1 + 0.3 * torch.randn(k * d, generator=g)).to(wtype or dtype).cuda() for k in n)
    pos = torch.stack([torch.randint(0, e, (B, T), generator=g) for e in extents], dim=-1).to(torch.int32).cuda()
    entries = sum(e * p for e, p in zip(extents, pairs))
    a = torch.rand(entries, generator=g) * 6.3
    tables = (a.cos().cuda(), a.sin().cuda(), extents, pairs)
    grads = [torch.randn(B, h, T, d, generator=g).to(dtype).cuda() for h in (H, KV, KV)]
    return qkv, qw, kw, pos, tables, grads


def split(qkv, H, KV, d):
    B, T, _ = qkv.shape
    x = lf.f64(qkv).view(B, T, H + 2 * KV, d)
    return x[:, :, :H], x[:, :, H:H + KV], x[:, :, H + KV:]


def parts(x, over):
    return (-2, -1) if over == "width" else (-1,)


def swap(a, pairs, halves):
    """Each rotated feature's partner in its place."""
    out, P = a.clone(), sum(pairs)
    for p in range(P):
        i, j = (p, P + p) if halves else (2 * p, 2 * p + 1)
        out[..., i], out[..., j] = a[..., j], a[..., i]
    rotated = torch.zeros(a.shape[-1], dtype=torch.bool)
    rotated[:2 * P] = True
    return torch.where(rotated, out, torch.zeros_like(out))


def check(B, T, H, KV, d, dtype, over, pairing, pairs, extents=(9, 5, 6), eps=1e-6, wtype=None, weights=True):
    from paper_2604_10103_b200 import layers
    qkv, qw, kw, pos, tables, grads = make(B, T, H, KV, d, dtype, over, extents, pairs, wtype=wtype)
    if not weights:
        qw = kw = None
    cos, sin = tables[:2]
    halves, u = pairing == "halves", lf.U[dtype]
    kws = dict(eps=eps, over=over, pairing=pairing)
    q, k, v = layers.split_heads_norm_rope(qkv, H, KV, qw, kw, pos, tables, **kws)
    dqkv, dqw, dkw = layers.split_heads_norm_rope_backward(*grads, qkv, qw, kw, pos, tables, **kws)
    again = layers.split_heads_norm_rope_backward(*grads, qkv, qw, kw, pos, tables, **kws)
    assert all(torch.equal(a, b) for a, b in zip((dqkv, dqw, dkw), again))
    xs = split(qkv, H, KV, d)
    assert torch.equal(v.transpose(1, 2).reshape(B, T, -1), qkv[..., (H + KV) * d:])
    out = lf.f64(dqkv).view(B, T, H + 2 * KV, d)
    assert torch.equal(out[:, :, H + KV:], lf.f64(grads[2]).transpose(1, 2))
    for name, x, got, w, dy, dgot, dw in (("q", xs[0], q, qw, grads[0], out[:, :, :H], dqw), ("k", xs[1], k, kw, grads[1], out[:, :, H:H + KV], dkw)):
        h = x.shape[2]
        n = d * (h if over == "width" else 1)
        wf = torch.ones(1, d, dtype=torch.float64) if w is None else lf.f64(w).view(-1, d)
        r = 1.0 / torch.sqrt(x.square().mean(parts(x, over), keepdim=True) + eps)
        xh = x * r
        ref = lf.rope(xh * wf, pos, cos, sin, extents, pairs, halves, False)
        a = (xh * wf).abs()
        lf.close(got.transpose(1, 2), ref, u * ref.abs() + lf.TINY[dtype] + (n / 2 + 16) * E * (a + swap(a, pairs, halves)), name)
        g = lf.rope(dy.transpose(1, 2), pos, cos, sin, extents, pairs, halves, True)
        ga = lf.f64(dy).transpose(1, 2).abs()
        ga = ga + swap(ga, pairs, halves)
        gw = g * wf
        mean = (gw * xh).mean(parts(x, over), keepdim=True)
        want = r * (gw - xh * mean)
        ea = r * (ga * wf.abs() + xh.abs() * (ga * wf.abs() * xh.abs()).mean(parts(x, over), keepdim=True))
        lf.close(dgot, want, u * want.abs() + lf.TINY[dtype] + (2 * n + 32) * E * ea, f"d{name}")
        over_axes = (0, 1) if over == "width" else (0, 1, 2)
        lf.close(dw, (g * xh).sum(over_axes).reshape(-1), (B * T * h + n + 32) * E * (ga * xh.abs()).sum(over_axes).reshape(-1) + 1e-40, f"d{name}_weight")


@pytest.mark.parametrize("T", [1, 2, 3, 31, 65, 130])
@pytest.mark.parametrize("over", ["head", "width"])
def test_tokens(T, over):
    check(1, T, 12, 12, 128, BF, over, "adjacent", (22, 21, 21))


@pytest.mark.parametrize("B,T,H,KV,d,pairs", [
    (2, 17, 2, 2, 64, (12, 10, 10)), (1, 40, 5, 5, 64, (12, 10, 10)), (2, 9, 8, 2, 64, (8, 8, 8)), (1, 33, 16, 4, 128, (24, 20, 20)),
    (1, 21, 24, 24, 128, (22, 21, 21)), (1, 7, 40, 8, 128, (22, 21, 21)), (1, 19, 10, 10, 96, (16, 16, 16)), (1, 12, 10, 5, 80, (4, 4, 4)),
    (3, 11, 3, 1, 256, (44, 42, 42)), (1, 5, 1, 1, 8, (2, 1, 1)), (1, 26, 4, 2, 10, (2, 2, 1)), (2, 13, 7, 7, 2, (1, 0, 0)), (1, 14, 6, 3, 38, (5, 5, 5)),
    (1, 3, 64, 64, 256, (44, 42, 42)), (1, 4, 130, 13, 64, (12, 10, 10)), (1, 6, 2048, 1, 8, (4, 0, 0))])
@pytest.mark.parametrize("dtype", [BF, F32, HALF])
def test_heads_widths_and_types(B, T, H, KV, d, pairs, dtype):
    for over, pairing in (("head", "halves"), ("width", "adjacent"), ("width", "halves"), ("head", "adjacent")):
        check(B, T, H, KV, d, dtype, over, pairing, pairs)


@pytest.mark.parametrize("H,KV,d,dtype", [(30, 20, 128, BF), (130, 70, 64, F32), (22, 14, 128, HALF), (9, 7, 250, BF)])
def test_shared_key_heads_that_leave_warps_idle(H, KV, d, dtype):
    for over, pairing in (("width", "adjacent"), ("head", "halves")):
        check(2, 45, H, KV, d, dtype, over, pairing, (8, 4, 4))


@pytest.mark.parametrize("over", ["head", "width"])
def test_weights_in_float32_and_none(over):
    check(2, 29, 6, 3, 64, BF, over, "adjacent", (12, 10, 10), wtype=F32)
    check(2, 29, 6, 3, 64, HALF, over, "halves", (12, 12, 8), wtype=F32)
    check(2, 29, 6, 3, 64, BF, over, "adjacent", (12, 10, 10), weights=False)
    check(1, 10, 6, 3, 62, BF, over, "adjacent", (12, 10, 9), wtype=F32)


def test_many_tokens():
    check(1, 3001, 4, 4, 64, BF, "width", "adjacent", (12, 10, 10))
    check(2, 1500, 3, 1, 40, F32, "head", "halves", (8, 4, 4))


def test_many_batches_of_few_tokens():
    """The walk over tokens passes several batches at a step."""
    for T in (1, 3):
        check(3001, T, 2, 1, 64, BF, "width", "adjacent", (12, 10, 10))
        check(1700, T, 2, 2, 64, BF, "head", "halves", (12, 10, 10))


@pytest.mark.parametrize("dtype,lead", [(BF, 8), (BF, 1), (F32, 3)])
@pytest.mark.parametrize("over", ["head", "width"])
def test_strides(dtype, lead, over):
    """Rows out of a wider tensor (on 16 bytes and off them), gradients token-major: the same bits as from contiguous ones."""
    from paper_2604_10103_b200 import layers
    qkv, qw, kw, pos, tables, grads = make(2, 21, 4, 2, 64, dtype, over, (9, 5, 6), (12, 10, 10))
    wide = torch.full((2, 21, qkv.shape[-1] + 24), float("nan"), dtype=dtype, device="cuda")
    wide[..., lead:lead + qkv.shape[-1]] = qkv
    view = wide[..., lead:lead + qkv.shape[-1]]
    turned = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in grads]
    a = layers.split_heads_norm_rope(qkv, 4, 2, qw, kw, pos, tables, over=over)
    b = layers.split_heads_norm_rope(view, 4, 2, qw, kw, pos, tables, over=over)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) or lead % 8
    for x, y in zip(a, b):
        assert lf.rel(x, lf.f64(y)) < 2 * lf.U[dtype]
    a = layers.split_heads_norm_rope_backward(*grads, qkv, qw, kw, pos, tables, over=over)
    b = layers.split_heads_norm_rope_backward(*turned, view, qw, kw, pos, tables, over=over)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) or lead % 8
    for x, y in zip(a, b):
        assert lf.rel(x, lf.f64(y)) < max(2 * lf.U[dtype], 200 * E)


def test_rows_of_zeros_and_values_that_are_not_finite():
    from paper_2604_10103_b200 import layers
    qkv, qw, kw, pos, tables, grads = make(1, 6, 4, 4, 64, BF, "head", (9, 5, 6), (12, 10, 10))
    qkv[0, 1] = 0
    qkv[0, 3, 64:128] = float("inf")        # head 1 of q, token 3
    for over in ("head", "width"):
        w = (qw, kw) if over == "head" else (qw.repeat(4), kw.repeat(4))
        q, k, v = layers.split_heads_norm_rope(qkv, 4, 4, *w, pos, tables, over=over)
        d, dqw, dkw = layers.split_heads_norm_rope_backward(*grads, qkv, *w, pos, tables, over=over)
        assert (q[0, :, 1] == 0).all() and (k[0, :, 1] == 0).all() and torch.isfinite(d[0, 1]).all()
        bad = ~torch.isfinite(q[0])
        assert bad[1, 3].any() and not bad[:, [0, 1, 2, 4, 5]].any() and (over == "width" or not bad[[0, 2, 3]].any())
        assert torch.isfinite(k).all() and torch.isfinite(v).all() and torch.isfinite(dkw).all()


def test_no_tokens():
    from paper_2604_10103_b200 import layers
    qkv, qw, kw, pos, tables, grads = make(1, 4, 4, 2, 64, BF, "width", (9, 5, 6), (12, 10, 10))
    q, k, v = layers.split_heads_norm_rope(qkv[:, :0], 4, 2, qw, kw, pos[:, :0], tables, over="width")
    assert q.shape == (1, 4, 0, 64) and v.shape == (1, 2, 0, 64)
    d, dqw, dkw = layers.split_heads_norm_rope_backward(q, k, v, qkv[:, :0], qw, kw, pos[:, :0], tables, over="width")
    assert d.shape == (1, 0, 512) and (dqw == 0).all() and (dkw == 0).all()


def test_a_position_outside_its_table_is_reported():
    from paper_2604_10103_b200 import binding as hf, layers
    qkv, qw, kw, pos, tables, grads = make(1, 8, 2, 2, 64, BF, "head", (9, 5, 6), (12, 10, 10))
    bad = pos.clone()
    bad[0, 5, 1] = 5
    zero = pos.clone()
    zero[0, 5, 1] = 0
    got = layers.split_heads_norm_rope(qkv, 2, 2, qw, kw, bad, tables)
    with pytest.raises(hf.HFError):
        hf.hf_layers_status()
    want = layers.split_heads_norm_rope(qkv, 2, 2, qw, kw, zero, tables)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    layers.split_heads_norm_rope_backward(*grads, qkv, qw, kw, bad, tables)
    with pytest.raises(hf.HFError):
        hf.hf_layers_status()


@pytest.mark.parametrize("over", ["head", "width"])
def test_autograd_and_differences(over):
    """Through torch's graph the same gradients; and they are the slopes of the 64-bit form: central differences along random directions, float32 inputs."""
    from paper_2604_10103_b200 import layers
    H, KV, d, pairs, extents = 4, 2, 32, (6, 5, 5), (9, 5, 6)
    qkv, qw, kw, pos, tables, grads = make(2, 9, H, KV, d, F32, over, extents, pairs)
    leaves = [t.clone().requires_grad_() for t in (qkv, qw, kw)]
    outs = layers.split_heads_norm_rope(leaves[0], H, KV, leaves[1], leaves[2], pos, tables, over=over)
    got = torch.autograd.grad(outs, leaves, grads)
    direct = layers.split_heads_norm_rope_backward(*grads, qkv, qw, kw, pos, tables, over=over)
    assert all(torch.equal(a, b) for a, b in zip(got, direct))

    def value(x, a, b):
        total = 0.0
        for xx, w, dy in zip(split(x, H, KV, d), (a, b, None), grads):
            dy = lf.f64(dy).transpose(1, 2)
            if w is None:
                total += (xx * dy).sum()
                continue
            r = 1.0 / torch.sqrt(xx.square().mean(parts(xx, over), keepdim=True) + 1e-6)
            total += (lf.rope(xx * r * lf.f64(w).view(-1, d), pos, *tables[:2], extents, pairs, False, False) * dy).sum()
        return total
    g = torch.Generator().manual_seed(3)
    base = [lf.f64(t) for t in (qkv, qw, kw)]
    for i in range(3):
        v = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
        h = 1e-6
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + h * v, base[i] - h * v
        slope = float(value(*up) - value(*down)) / (2 * h)
        mine = float((lf.f64(got[i]) * v).sum())
        assert abs(slope - mine) < 1e-4 * float((lf.f64(got[i]) * v).abs().sum()) + 1e-6


def test_captured_on_another_stream():
    from paper_2604_10103_b200 import layers
    qkv, qw, kw, pos, tables, grads = make(1, 50, 12, 12, 128, BF, "width", (9, 5, 6), (22, 21, 21))
    want = layers.split_heads_norm_rope(qkv, 12, 12, qw, kw, pos, tables, over="width")
    dwant = layers.split_heads_norm_rope_backward(*grads, qkv, qw, kw, pos, tables, over="width")
    g = torch.cuda.CUDAGraph()
    static = torch.zeros_like(qkv)
    with torch.cuda.graph(g):
        got = layers.split_heads_norm_rope(static, 12, 12, qw, kw, pos, tables, over="width")
        dgot = layers.split_heads_norm_rope_backward(*grads, static, qw, kw, pos, tables, over="width")
    static.copy_(qkv)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + dwant, got + dgot))
