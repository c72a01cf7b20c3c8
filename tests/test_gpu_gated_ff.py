"""Gated feed-forward and its gradients against the definition in 64 bits.

Bounds.  The forward rounds h once (U |h|) and y once; g and u carry a float32 sum's error of width 2^-24 of the absolute terms, which
act and the product pass on with factors below 1.2 and |u|.  Element by element that is U |y| + (U + ...) sum |h| |Wd|, and in the 2-norm
two independent roundings of relative size at most U / sqrt(3) each stay below U.  The backward pass rounds dg, du, h once and each
result once: the same two roundings."""
import ctypes as C

import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def no_wait_ran_out():
    """A bounded wait that runs out may leave right numbers behind: the status word tells."""
    yield
    from paper_2604_10103_b200 import binding as hf
    assert hf.hf_layers_status() == (0, 0)


BF, HALF = torch.bfloat16, torch.float16


def make(M, K, N, O, dtype, seed=0):
    g = torch.Generator().manual_seed(M * 31 + K * 7 + N + seed)
    x = torch.randn(M, K, generator=g)
    wg, wu = 1.5 * torch.randn(N, K, generator=g) / K ** 0.5, torch.randn(N, K, generator=g) / K ** 0.5
    wd, dy = torch.randn(O, N, generator=g) / N ** 0.5, torch.randn(M, O, generator=g)
    return [t.to(dtype).cuda() for t in (x, wg, wu, wd, dy)]


def check(M, K, N, O, dtype, act, seed=0):
    from paper_2604_10103_b200 import layers
    x, wg, wu, wd, dy = make(M, K, N, O, dtype, seed)
    u = lf.U[dtype]
    y, gate, up = layers.gated_ff(x, wg, wu, wd, act=act, save=True)
    ry, rg, ru, rh = lf.ff(x, wg, wu, wd, act)
    ex = 2.0 ** -24 * (K + 16)
    ag, au = lf.f64(x).abs() @ lf.f64(wg).abs().t(), lf.f64(x).abs() @ lf.f64(wu).abs().t()
    lf.close(gate, rg, u * rg.abs() + lf.TINY[dtype] + ex * ag, "gate")
    lf.close(up, ru, u * ru.abs() + lf.TINY[dtype] + ex * au, "up")
    eh = u * rh.abs() + lf.TINY[dtype] + 1.2 * ex * ag * ru.abs() + (rg.abs() + 0.2) * ex * au + 16 * 2.0 ** -24 * rh.abs()
    sums = lf.f64(wd).abs()
    lf.close(y, ry, u * ry.abs() + lf.TINY[dtype] + (1 + u) * (eh @ sums.t()) + 2.0 ** -24 * (N + 16) * (rh.abs() @ sums.t()), "y")
    if M * O >= 64:
        assert lf.rel(y, ry) < u
    assert torch.equal(layers.gated_ff(x, wg, wu, wd, act=act), y)
    got = layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up, act=act)
    *ref, rdg, rdu, rh2 = lf.ff_backward(dy, x, wg, wu, wd, gate, up, act)
    adh = lf.f64(dy).abs() @ sums
    # float32 error of dh, times |u| act' (at most 1.2 |u|) or act
    e32 = 2.0 ** -24 * (O + 32)
    edg = u * rdg.abs() + lf.TINY[dtype] + e32 * adh * 1.2 * lf.f64(up).abs()
    edu = u * rdu.abs() + lf.TINY[dtype] + e32 * adh * (lf.f64(gate).abs() + 0.2)
    ehb = u * rh2.abs() + lf.TINY[dtype] + 32 * 2.0 ** -24 * rh2.abs()
    w_g, w_u, ax = lf.f64(wg).abs(), lf.f64(wu).abs(), lf.f64(x).abs()
    s = 1 + u
    bounds = (s * (edg @ w_g + edu @ w_u) + 2.0 ** -24 * (2 * N + 16) * (rdg.abs() @ w_g + rdu.abs() @ w_u),
              s * (edg.t() @ ax) + 2.0 ** -24 * (M + 16) * (rdg.abs().t() @ ax),
              s * (edu.t() @ ax) + 2.0 ** -24 * (M + 16) * (rdu.abs().t() @ ax),
              s * (lf.f64(dy).abs().t() @ ehb) + 2.0 ** -24 * (M + 16) * (lf.f64(dy).abs().t() @ rh2.abs()))
    for name, p, r, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, ref, bounds):
        lf.close(p, r, u * r.abs() + lf.TINY[dtype] + b, name)
        if r.numel() >= 64:
            assert lf.rel(p, r) < u, name
    again = layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up, act=act)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 255, 257, 400])
def test_rows(M):
    check(M, 264, 520, 264, BF, "silu")


@pytest.mark.parametrize("M,K,N,O", [(1, 8, 8, 8), (3, 8, 16, 24), (70, 64, 64, 64), (130, 72, 24, 200), (50, 1536, 1368, 1536), (200, 136, 2048, 40),
                                     (300, 40, 8, 3000), (1000, 648, 1304, 648), (129, 512, 4104, 520)])
@pytest.mark.parametrize("dtype,act", [(BF, "silu"), (HALF, "gelu_tanh"), (BF, "gelu_tanh"), (HALF, "silu")])
def test_widths_types_and_activations(M, K, N, O, dtype, act):
    check(M, K, N, O, dtype, act)


@pytest.mark.parametrize("M", [1, 5, 600])
def test_the_832x480_width(M):
    check(M, 1536, 4096, 1536, BF, "silu")


def test_long_contractions_over_rows():
    """Few weights and many rows: the contraction of dW is long."""
    check(9000, 64, 136, 64, BF, "silu")


@pytest.mark.parametrize("M", [3, 90, 260])
def test_strided_rows(M):
    from paper_2604_10103_b200 import layers
    x, wg, wu, wd, dy = make(M, 256, 512, 128, BF)
    xs = torch.full((M, 3 * 256), float("nan"), dtype=BF, device="cuda")
    xs[:, 256:512] = x
    dys = torch.full((M, 136), float("nan"), dtype=BF, device="cuda")
    dys[:, 8:] = dy
    y, g, u = layers.gated_ff(x, wg, wu, wd, save=True)
    y2, g2, u2 = layers.gated_ff(xs[:, 256:512], wg, wu, wd, save=True)
    assert torch.equal(y, y2) and torch.equal(g, g2) and torch.equal(u, u2)
    a = layers.gated_ff_backward(dy, x, wg, wu, wd, g, u)
    b = layers.gated_ff_backward(dys[:, 8:], xs[:, 256:512], wg, wu, wd, g, u)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    y3 = layers.gated_ff(x.view(1, M, 256), wg, wu, wd)
    assert y3.shape == (1, M, 128) and torch.equal(y3[0], y)


def test_gradients_against_differences():
    """Directional central differences of the 64-bit forward; the saved projections are rounded (U each), so are dg, du, h and the result."""
    from paper_2604_10103_b200 import layers
    M, K, N, O, h = 40, 96, 160, 96, 1e-5
    for act in ("silu", "gelu_tanh"):
        x, wg, wu, wd, dy = make(M, K, N, O, HALF)
        _, gate, up = layers.gated_ff(x, wg, wu, wd, act=act, save=True)
        grads = layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up, act=act)
        gen = torch.Generator().manual_seed(3)
        args = [lf.f64(t) for t in (x, wg, wu, wd)]
        for which, grad in enumerate(grads):
            v = torch.randn(args[which].shape, generator=gen, dtype=torch.float64)
            ends = []
            for s in (1, -1):
                moved = list(args)
                moved[which] = args[which] + s * h * v
                ends.append((lf.ff(*moved, act)[0] * lf.f64(dy)).sum())
            diff, got = float(ends[0] - ends[1]) / (2 * h), float((lf.f64(grad) * v).sum())
            assert abs(got - diff) <= 6 * lf.U[HALF] * float((lf.f64(grad) * v).norm()) + 1e-6 * float((lf.f64(grad) * v).abs().sum()), (act, which)


@pytest.mark.parametrize("M", [5, 200])
def test_saturated_activations(M):
    """Gates far out on both sides: act is 0 or g, its slope 0 or 1, and nothing overflows on the way."""
    from paper_2604_10103_b200 import layers
    K = N = O = 128
    x, wg, wu, wd, dy = make(M, K, N, O, BF)
    x[: M // 2] *= 200.0
    for act in ("silu", "gelu_tanh"):
        y, gate, up = layers.gated_ff(x, wg, wu, wd, act=act, save=True)
        assert lf.rel(y, lf.ff(x, wg, wu, wd, act)[0]) < lf.U[BF]
        for p, r in zip(layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up, act=act), lf.ff_backward(dy, x, wg, wu, wd, gate, up, act)):
            assert lf.rel(p, r) < lf.U[BF]


@pytest.mark.parametrize("M", [6, 150])
def test_a_row_of_nan_stays_alone(M):
    from paper_2604_10103_b200 import layers
    x, wg, wu, wd, dy = make(M, 136, 264, 136, BF)
    y, gate, up = layers.gated_ff(x, wg, wu, wd, save=True)
    bad = x.clone()
    bad[M - 1, 5] = float("nan")
    y2, gate2, up2 = layers.gated_ff(bad, wg, wu, wd, save=True)
    assert torch.equal(y[:-1], y2[:-1]) and torch.isnan(y2[-1]).all()
    dx = layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up)[0]
    dx2 = layers.gated_ff_backward(dy, bad, wg, wu, wd, gate2, up2)[0]
    assert torch.equal(dx[:-1], dx2[:-1]) and torch.isnan(dx2[-1]).all()


def test_no_rows():
    from paper_2604_10103_b200 import layers
    x, wg, wu, wd, dy = make(4, 64, 128, 64, BF)
    y, g, u = layers.gated_ff(x[:0], wg, wu, wd, save=True)
    assert y.shape == (0, 64) and g.shape == (0, 128)
    dx, *dw = layers.gated_ff_backward(dy[:0], x[:0], wg, wu, wd, g, u)
    assert dx.shape == (0, 64) and all(not t.any() for t in dw)


@pytest.mark.parametrize("M", [2, 300])
def test_another_stream_and_a_graph(M):
    from paper_2604_10103_b200 import binding as hf, layers
    x, wg, wu, wd, dy = make(M, 512, 1024, 512, BF)

    def both():
        y, g, u = layers.gated_ff(x, wg, wu, wd, save=True)
        return (y, g, u) + layers.gated_ff_backward(dy, x, wg, wu, wd, g, u)
    ref = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = both()
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for t in got:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    assert hf.hf_layers_status() == (0, 0)


def test_nothing_is_written_past_the_outputs():
    """Ragged sizes: canaries behind every output, and the workspace's own end."""
    from paper_2604_10103_b200 import binding as hf, layers
    for M in (5, 130):
        K, N, O = 72, 136, 104
        x, wg, wu, wd, dy = make(M, K, N, O, BF)
        s = hf.hf_ff_shape(type=0, act=0, rows=M, width=K, hidden=N, out_width=O, x_stride=K, y_stride=O)

        def guarded(n):
            return torch.full((n + 512,), 7.0, dtype=BF, device="cuda")
        sizes = dict(y=M * O, gate=M * N, up=M * N, dx=M * K, dwg=N * K, dwu=N * K, dwd=O * N)
        b = {k: guarded(n) for k, n in sizes.items()}
        ws = [torch.full((hf.hf_gated_ff_workspace(C.byref(s), k) + 1024,), 99, dtype=torch.uint8, device="cuda") for k in (0, 1)]
        hf.hf_gated_ff(C.byref(s), x, wg, wu, wd, b["y"], b["gate"], b["up"], ws[0])
        hf.hf_gated_ff_backward(C.byref(s), dy, x, wg, wu, wd, b["gate"], b["up"], b["dx"], b["dwg"], b["dwu"], b["dwd"], ws[1])
        torch.cuda.synchronize()
        for k, n in sizes.items():
            assert (b[k][n:] == 7.0).all(), k
        assert all((w[-1024:] == 99).all() for w in ws)
        y, gate, up = layers.gated_ff(x, wg, wu, wd, save=True)
        assert torch.equal(b["y"][:M * O].view(M, O), y) and torch.equal(b["up"][:M * N].view(M, N), up)
        # dx alone, and the weights' gradients alone
        dx = guarded(M * K)
        hf.hf_gated_ff_backward(C.byref(s), dy, x, wg, wu, wd, gate, up, dx, None, None, None, ws[1])
        assert torch.equal(dx, b["dx"])
        d3 = [guarded(n) for n in (N * K, N * K, O * N)]
        hf.hf_gated_ff_backward(C.byref(s), dy, x, wg, wu, wd, gate, up, None, *d3, ws[1])
        assert all(torch.equal(p, b[k]) for p, k in zip(d3, ("dwg", "dwu", "dwd")))
