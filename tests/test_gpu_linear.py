"""Linear layers with bias, activation, gate and residual, and their gradients, against the definition in 64 bits.

Bounds.  The sums carry a float32 error of (K + 16) 2^-24 of their absolute terms, which the activation passes on with a factor below 1.2, plus 16 2^-24
of its own value; the gate's product and the residual's sum round once each, the result once more (U |y|).  The backward pass rounds dp once (U |dp|)
and each product once; db and dgate are float32 sums of dp before its rounding."""
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32
E = 2.0 ** -24


@pytest.fixture(autouse=True)
def no_wait_ran_out():
    yield
    from paper_2604_10103_b200 import binding as hf
    assert hf.hf_layers_status() == (0, 0)


def make(M, K, N, dtype, bias=True, group=0, residual=True, seed=0, ptype=None):
    g = torch.Generator().manual_seed(M * 31 + K * 7 + N + seed)
    x, w = torch.randn(M, K, generator=g), torch.randn(N, K, generator=g) / K ** 0.5
    dy, res = torch.randn(M, N, generator=g), torch.randn(M, N, generator=g)
    b = torch.randn(N, generator=g).to(ptype or dtype).cuda() if bias else None
    gate = torch.randn(-(-M // group) if group > 0 else 1, N, generator=g).to(ptype or dtype).cuda() if group else None       # (group -1: one row)
    x, w, dy, res = (t.to(dtype).cuda() for t in (x, w, dy, res))
    return x, w, b, gate, res if residual else None, dy


def acts(p, name):
    return p if name is None else lf.act(p, name)


def check(M, K, N, dtype, act=None, bias=True, group=0, residual=True, ptype=None):
    from paper_2604_10103_b200 import layers
    x, w, b, gate, res, dy = make(M, K, N, dtype, bias, group, residual, ptype=ptype)
    kw, u, tiny = dict(act=act, gate=gate, rows_per_group=max(group, 0)), lf.U[dtype], lf.TINY[dtype]
    y, pre = layers.linear(x, w, b, residual=res, save=True, **kw)
    fx, fw = lf.f64(x), lf.f64(w)
    of = lf.groups_of(M, max(group, 0))
    gf = torch.ones(1, N, dtype=torch.float64) if gate is None else lf.f64(gate).view(-1, N)
    rp = fx @ fw.t() + (0.0 if b is None else lf.f64(b))
    ep = E * (K + 16) * (fx.abs() @ fw.abs().t() + (0.0 if b is None else lf.f64(b).abs()))
    lf.close(pre, rp, u * rp.abs() + tiny + ep, "pre")
    ra = acts(rp, act)
    ry = ra * gf[of] + (0.0 if res is None else lf.f64(res))
    ey = (1.2 * ep + 16 * E * ra.abs()) * gf[of].abs() + 4 * E * (ry.abs() + ra.abs() * gf[of].abs())
    lf.close(y, ry, u * ry.abs() + tiny + (1 + u) * ey, "y")
    assert torch.equal(layers.linear(x, w, b, residual=res, **kw), y)
    saved = pre if act is not None or gate is not None else None
    got = layers.linear_backward(dy, x, w, saved, **kw)
    p = lf.f64(pre).requires_grad_()
    a = acts(p, act)
    fd = lf.f64(dy)
    slope = torch.autograd.grad(a.sum(), p)[0]
    a = a.detach()
    dp = fd * gf[of] * slope
    e32 = 40 * E * (fd * gf[of]).abs() * (slope.abs() + 0.1 if act else 0.0)
    edp = (u * dp.abs() + tiny if saved is not None else 0.0) + e32
    lf.close(got[0], dp @ fw, u * (dp @ fw).abs() + tiny + (1 + u) * (edp @ fw.abs() if torch.is_tensor(edp) else 0.0) + E * (N + 16) * (dp.abs() @ fw.abs()), "dx")
    lf.close(got[1], dp.t() @ fx, u * (dp.t() @ fx).abs() + tiny + (1 + u) * (edp.t() @ fx.abs() if torch.is_tensor(edp) else 0.0) + E * (M + 16) * (dp.abs().t() @ fx.abs()), "dweight")
    lf.close(got[2], dp.sum(0), (e32.sum(0) if torch.is_tensor(e32) else 0.0) + E * (M + 16) * dp.abs().sum(0) + 1e-40, "dbias")
    if gate is None:
        assert got[3] is None
    else:
        t = fd * a
        zero = torch.zeros(gf.shape, dtype=torch.float64)
        lf.close(got[3], zero.index_add(0, of, t), E * (M + 40) * zero.index_add(0, of, t.abs()) + 1e-40, "dgate")
    again = layers.linear_backward(dy, x, w, saved, **kw)
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 127, 129, 255, 257, 400])
def test_rows(M):
    check(M, 264, 520, BF, "silu", group=max(1, M // 3))


@pytest.mark.parametrize("M,K,N", [(1, 8, 8), (3, 8, 24), (70, 64, 64), (130, 72, 200), (50, 1536, 1368), (200, 136, 40), (300, 40, 3000), (1000, 648, 648),
                                   (129, 4104, 520), (5, 1544, 9224), (14, 6152, 1536), (2, 264, 8200)])
@pytest.mark.parametrize("dtype,act,bias,group,residual", [(BF, None, True, 0, False), (HALF, "gelu_tanh", True, 7, True), (BF, "gelu_tanh", False, -1, False),
                                                           (HALF, "silu", False, 0, True), (BF, None, False, 0, False), (BF, None, True, 1, True)])
def test_widths_types_and_epilogues(M, K, N, dtype, act, bias, group, residual):
    check(M, K, N, dtype, act, bias, group, residual)


@pytest.mark.parametrize("M", [1, 20, 500])
def test_parameters_in_float32(M):
    check(M, 200, 328, BF, "silu", group=max(1, M // 4), ptype=F32)
    check(M, 200, 328, HALF, None, group=0, residual=False, ptype=F32)


@pytest.mark.parametrize("M", [1, 5, 600])
def test_the_832x480_widths(M):
    check(M, 1536, 6144, BF, "gelu_tanh", residual=False)
    check(M, 6144, 1536, BF, None, group=200)


def test_long_contractions_over_rows_and_many_groups():
    check(9000, 64, 136, BF, "silu", group=1560)
    check(3000, 64, 72, BF, None, group=1)


@pytest.mark.parametrize("M", [3, 90, 260])
def test_strided_rows_and_slices(M):
    from paper_2604_10103_b200 import layers
    x, w, b, gate, res, dy = make(M, 256, 512, BF, group=40)

    def strided(t, before, after):
        s = torch.full((t.shape[0], before + t.shape[1] + after), float("nan"), dtype=BF, device="cuda")
        s[:, before:before + t.shape[1]] = t
        return s[:, before:before + t.shape[1]]
    xs, rs, ds, gs = strided(x, 256, 256), strided(res, 8, 0), strided(dy, 0, 16), strided(gate, 512, 1024)
    kw = dict(act="silu", rows_per_group=40)
    y, pre = layers.linear(x, w, b, gate=gate, residual=res, save=True, **kw)
    y2, pre2 = layers.linear(xs, w, b, gate=gs, residual=rs, save=True, **kw)
    assert torch.equal(y, y2) and torch.equal(pre, pre2)
    a = layers.linear_backward(dy, x, w, pre, gate=gate, **kw)
    c = layers.linear_backward(ds, xs, w, pre, gate=gs, **kw)
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    y3 = layers.linear(x.view(1, M, 256), w, b, gate=gate, residual=res.view(1, M, 512), **kw)
    assert y3.shape == (1, M, 512) and torch.equal(y3[0], y)


def test_only_what_is_asked_for():
    from paper_2604_10103_b200 import layers
    x, w, b, gate, res, dy = make(100, 64, 128, BF, group=30)
    _, pre = layers.linear(x, w, b, act="silu", gate=gate, rows_per_group=30, save=True)
    full = layers.linear_backward(dy, x, w, pre, "silu", gate, 30)
    for i, name in enumerate(("dx", "dweight", "dbias", "dgate")):
        got = layers.linear_backward(dy, x, w, pre, "silu", gate, 30, **{k: k == name for k in ("dx", "dweight", "dbias", "dgate")})
        assert torch.equal(got[i], full[i]) and all(t is None for j, t in enumerate(got) if j != i)


@pytest.mark.parametrize("M", [3, 200])
def test_values_that_are_not_finite_stay_in_their_rows(M):
    from paper_2604_10103_b200 import layers
    x, w, b, gate, res, dy = make(M, 128, 256, BF, group=1)
    clean = layers.linear(x, w, b, act="silu", gate=gate, residual=res, rows_per_group=1)
    x[1, 5], res[2, 9] = float("nan"), float("inf")
    gate[0] = 0.0
    y = layers.linear(x, w, b, act="silu", gate=gate, residual=res, rows_per_group=1)
    assert torch.isnan(y[1]).all() and torch.isinf(y[2, 9]) and torch.equal(y[0], res[0]) and torch.equal(y[3:], clean[3:])
    assert torch.equal(y[2, :9], clean[2, :9]) and torch.equal(y[2, 10:], clean[2, 10:])


def test_gates_far_out():
    """silu and gelu far on both sides: 0 and the value itself, slopes 0 and 1."""
    from paper_2604_10103_b200 import layers
    for act in ("silu", "gelu_tanh"):
        b = torch.tensor([-3e38, -1e20, -200.0, 200.0, 1e20, 3e38, 0.0, 1.0], device="cuda")
        for M in (2, 40):
            x, w = torch.zeros(M, 8, dtype=BF, device="cuda"), torch.zeros(8, 8, dtype=BF, device="cuda")
            y, pre = layers.linear(x, w, b, act=act, save=True)
            want = torch.where(b < -100, torch.zeros_like(b), torch.where(b > 100, b, y[0].float()))
            assert torch.equal(y.float(), want.to(BF).float().expand(M, 8))
            db = layers.linear_backward(torch.ones(M, 8, dtype=BF, device="cuda"), x, w, pre, act)[2]
            assert torch.equal(db[:6], M * (b[:6] > 0).float())


def test_no_rows():
    from paper_2604_10103_b200 import layers
    x, w, b, gate, res, dy = make(4, 64, 128, BF, group=2)
    y, pre = layers.linear(x[:0], w, b, act="silu", gate=gate[:0], residual=res[:0], rows_per_group=2, save=True)
    assert y.shape == (0, 128) and pre.shape == (0, 128)
    dx, dw, db, dg = layers.linear_backward(dy[:0], x[:0], w, pre, "silu", gate[:0], 2)
    assert dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all() and dg.shape == (0, 128)


def test_autograd_is_the_backward_call():
    from paper_2604_10103_b200 import layers
    for act, group, bias, residual in (("gelu_tanh", 30, True, True), (None, 0, True, False), (None, 0, False, True), ("silu", 0, False, False)):
        x, w, b, gate, res, dy = make(90, 64, 128, BF, bias, group, residual)
        leaves = [t for t in (x, w, b, gate, res) if t is not None]
        for t in leaves:
            t.requires_grad_()
        y = layers.linear(x, w, b, act=act, gate=gate, residual=res, rows_per_group=group)
        got = torch.autograd.grad(y, leaves, dy)
        with torch.no_grad():
            _, pre = layers.linear(x, w, b, act=act, gate=gate, residual=res, rows_per_group=group, save=True)
            dx, dw, db, dg = layers.linear_backward(dy, x, w, pre, act, gate, group)
        want = [t for t, leaf in ((dx, x), (dw, w), (db.to(BF), b), (None if dg is None else dg.to(BF), gate), (dy, res)) if leaf is not None]
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_gradients_against_differences():
    """Directional central differences of the 64-bit forward; pre, dp and the results are rounded (U each, of a sum of absolute terms)."""
    from paper_2604_10103_b200 import layers
    M, K, N, h = 40, 96, 160, 1e-5
    for act in (None, "silu", "gelu_tanh"):
        x, w, b, gate, res, dy = make(M, K, N, HALF, group=9)
        _, pre = layers.linear(x, w, b, act=act, gate=gate, residual=res, rows_per_group=9, save=True)
        got = layers.linear_backward(dy, x, w, pre, act, gate, 9)
        of = lf.groups_of(M, 9)

        def value(x, w, b, gate):
            return ((acts(x @ w.t() + b, act) * gate[of]) * lf.f64(dy)).sum()
        base = [lf.f64(t) for t in (x, w, b, gate)]
        g = torch.Generator().manual_seed(1)
        for i in range(4):
            v = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
            up, down = list(base), list(base)
            up[i], down[i] = base[i] + h * v, base[i] - h * v
            slope = float(value(*up) - value(*down)) / (2 * h)
            terms = lf.f64(got[i]) * v
            # independent roundings: their sum's standard deviation is below U of the terms' 2-norm, times the three of them; six of those
            assert abs(slope - float(terms.sum())) < 6 * 3 * lf.U[HALF] * float(terms.norm()) * 3


def test_first_call_captured_and_replayed_with_other_values():
    from paper_2604_10103_b200 import layers
    x, w, b, gate, res, dy = make(300, 256, 264, BF, group=100)
    layers.linear(x[:20], w, b)
    static = torch.zeros_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, pre = layers.linear(static, w, b, act="silu", gate=gate, residual=res, rows_per_group=100, save=True)
        grads = layers.linear_backward(dy, static, w, pre, "silu", gate, 100)
    static.copy_(x)
    g.replay()
    wy, wpre = layers.linear(x, w, b, act="silu", gate=gate, residual=res, rows_per_group=100, save=True)
    want = layers.linear_backward(dy, x, w, wpre, "silu", gate, 100)
    assert torch.equal(y, wy) and torch.equal(pre, wpre) and all(torch.equal(p, q) for p, q in zip(grads, want))


def test_two_streams_at_once():
    from paper_2604_10103_b200 import layers
    a, c = make(2000, 512, 1024, BF, group=500, seed=1), make(700, 1024, 512, BF, seed=2)

    def once(t, group):
        y, pre = layers.linear(t[0], t[1], t[2], act="silu", gate=t[3], residual=t[4], rows_per_group=group, save=True)
        return (y, *layers.linear_backward(t[5], t[0], t[1], pre, "silu", t[3], group))
    want = once(a, 500), once(c, 0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = []
        for s, t, group in zip(streams, (a, c), (500, 0)):
            with torch.cuda.stream(s):
                got.append(once(t, group))
        torch.cuda.synchronize()
        for p, q in zip(want, got):
            assert all(m is n is None or torch.equal(m, n) for m, n in zip(p, q))
