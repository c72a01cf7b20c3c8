"""Layer norm and its gradients against the definition in 64 bits."""
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


BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


def make(rows, width, dtype, group=0, seed=0, param=None, shift=0.5):
    g = torch.Generator().manual_seed(1000 * rows + width + seed)
    groups = -(-rows // group) if group else 1
    x = (torch.randn(rows, width, generator=g) * torch.exp(0.5 * torch.randn(width, generator=g)) + shift).to(dtype).cuda()
    w = (0.3 * torch.randn(groups, width, generator=g)).to(param or dtype).cuda()
    b = (0.3 * torch.randn(groups, width, generator=g)).to(param or dtype).cuda()
    dy = torch.randn(rows, width, generator=g).to(dtype).cuda()
    return x, w, b, dy


def forward_bound(x, y, xhat, a, b_abs, rstd, dtype):
    """The mean is off by at most (D + 1) 2^-24 mean |x| and so is every difference; rstd relatively by (D + 4) 2^-24 and the difference's
    share; two more roundings.  Sums run over threads and a tree, so D / 8 + 32 terms follow one another at most."""
    n = x.shape[1] / 8 + 40
    e = n * 2.0 ** -24
    x = lf.f64(x)
    return lf.U[dtype] * y.abs() * (1 + e) + lf.TINY[dtype] + e * (a.abs() * (xhat.abs() * 3 + x.abs().mean(1, keepdim=True) * rstd[:, None] * (3 + xhat.abs())) + y.abs() + b_abs)


SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (2, 255), (4, 256), (9, 257), (17, 1000), (7, 1024), (33, 1536), (4, 2048), (3, 2056), (3, 4095),
          (2, 4104), (2, 8192), (2, 16384), (1, 16383), (300, 24)]


@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("rows,width", SHAPES)
def test_forward_and_backward(rows, width, dtype):
    from paper_2604_10103_b200 import layers
    for group, offset in ((0, 0.0), (max(1, rows // 3), 1.0)):
        x, w, b, dy = make(rows, width, dtype, group)
        eps = 1e-5
        y, mean, rstd = layers.layer_norm(x, w, b, eps=eps, weight_offset=offset, rows_per_group=group)
        ry, rmean, rrstd, xhat, a = lf.norm(x, w, b, eps, offset, group)
        bound = forward_bound(x, ry, xhat, a, lf.f64(b).abs().max(), rrstd, dtype)
        lf.close(y, ry, bound, "y")
        n = (width / 8 + 40) * 2.0 ** -24
        lf.close(mean, rmean, n * lf.f64(x).abs().mean(1), "mean")
        lf.close(rstd, rrstd, n * rrstd * (3 + 2 * lf.f64(x).abs().mean(1) * rrstd), "rstd")
        dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w, weight_offset=offset, rows_per_group=group)
        rdx, rdw, rdb, adw, adb = lf.norm_backward(dy, x, mean, rstd, w, offset, group)
        gh = (lf.f64(dy) * a).abs()
        scale = lf.f64(rstd)[:, None] * (gh + gh.mean(1, keepdim=True) + xhat.abs() * (gh * xhat.abs()).mean(1, keepdim=True))
        # (xhat is formed from the rounded difference: its absolute error is 2^-24 of |x| rstd)
        cancel = lf.f64(x).abs() * lf.f64(rstd)[:, None]
        extra = lf.f64(rstd)[:, None] * ((gh * cancel).mean(1, keepdim=True) * xhat.abs() + cancel * (gh * xhat.abs()).mean(1, keepdim=True))
        lf.close(dx, rdx, lf.U[dtype] * rdx.abs() + lf.TINY[dtype] + n * (scale + extra), "dx")
        m = (rows + 8) * 2.0 ** -24
        of = lf.groups_of(rows, group)
        acancel = torch.zeros_like(adw).index_add_(0, of, lf.f64(dy).abs() * cancel)
        lf.close(dw, rdw, m * adw + 4 * 2.0 ** -24 * acancel, "dw")
        lf.close(db, rdb, m * adb, "db")


@pytest.mark.parametrize("rows,width,group", [(4681, 1536, 0), (1200, 200, 7), (700, 96, 1), (2500, 1027, 1249)])
def test_many_rows_and_groups(rows, width, group):
    from paper_2604_10103_b200 import layers
    x, w, b, dy = make(rows, width, F32, group)
    y, mean, rstd = layers.layer_norm(x, w, b, weight_offset=1.0, rows_per_group=group)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w, weight_offset=1.0, rows_per_group=group)
    rdx, rdw, rdb, adw, adb = lf.norm_backward(dy, x, mean, rstd, w, 1.0, group)
    # rows are added in a few hundred partial sums of at most `rows` / 16 rows each
    lf.close(db, rdb, (rows / 16 + 64) * 2.0 ** -24 * adb, "db")
    assert lf.rel(dw, rdw) < 1e-5 and lf.rel(dx, rdx) < 1e-5 and lf.rel(y, lf.norm(x, w, b, 1e-6, 1.0, group)[0]) < 1e-5
    again = layers.layer_norm_backward(dy, x, mean, rstd, w, weight_offset=1.0, rows_per_group=group)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("param", [BF, F32])
def test_strided_rows_slices_of_a_modulation_tensor_and_parameter_types(param):
    from paper_2604_10103_b200 import layers
    rows, width, group = 30, 384, 10
    x, w, b, dy = make(rows, width, BF, group, param=param)
    wide = torch.zeros(rows, 3 * width, dtype=BF, device="cuda")
    wide[:, width:2 * width] = x
    mod = torch.zeros(3, 6, width, dtype=param, device="cuda")
    mod[:, 4], mod[:, 3] = w, b
    ref = layers.layer_norm(x, w, b, weight_offset=1.0, rows_per_group=group)
    got = layers.layer_norm(wide[:, width:2 * width], mod[:, 4], mod[:, 3], weight_offset=1.0, rows_per_group=group)
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    rb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w, weight_offset=1.0, rows_per_group=group)
    dyw = torch.zeros(rows, 2 * width, dtype=BF, device="cuda")
    dyw[:, :width] = dy
    gb = layers.layer_norm_backward(dyw[:, :width], wide[:, width:2 * width], ref[1], ref[2], mod[:, 4], weight_offset=1.0, rows_per_group=group)
    assert all(torch.equal(p, q) for p, q in zip(rb, gb))
    # one element off the 16-byte boundary: the other accesses, results equal up to the order of the sums
    off = torch.zeros(rows * width + 1, dtype=BF, device="cuda")[1:].view(rows, width)
    off.copy_(x)
    y1 = layers.layer_norm(off, w, b, weight_offset=1.0, rows_per_group=group)
    bound = lf.norm(x, w, b, 1e-6, 1.0, group)
    lf.close(y1[0], bound[0], forward_bound(x, bound[0], bound[3], bound[4], 2.0, bound[2], BF), "y of unaligned rows")


@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("width", [6, 31, 96, 641, 1454, 2167])
def test_rows_that_start_anywhere(width, dtype):
    """Every offset of x's, dy's and the parameters' first element within 16 bytes, and row strides that are no multiple of it."""
    from paper_2604_10103_b200 import layers
    rows = 29
    x, w, b, dy = make(rows, width, dtype)

    def moved(t, off, pad):
        m = torch.full((t.shape[0] * (width + pad) + off + 1,), float("nan"), dtype=t.dtype, device="cuda")
        v = m[off:off + t.shape[0] * (width + pad)].view(t.shape[0], width + pad)[:, :width]
        v.copy_(t)
        return v
    ry, rmean, rrstd, xhat, a = lf.norm(x, w, b, 1e-6, 0.0, 0)
    bound = forward_bound(x, ry, xhat, a, lf.f64(b).abs().max(), rrstd, dtype)
    for off, pad in ((0, 1), (1, 0), (2, 2), (3, 5), (4, 4), (5, 3), (6, 0), (7, 7)):
        xm, dm, wm, bm = moved(x, off, pad), moved(dy, (3 * off + 1) % 8, pad + 1), moved(w, (off + 2) % 8, 0), moved(b, (off + 2) % 8, 0)
        y, mean, rstd = layers.layer_norm(xm, wm, bm)
        lf.close(y, ry, bound, f"y at {off}, {pad}")
        dx, dw, db = layers.layer_norm_backward(dm, xm, mean, rstd, wm)
        rdx, rdw, rdb, adw, adb = lf.norm_backward(dy, x, mean, rstd, w, 0.0, 0)
        lf.close(db, rdb, (rows + 8) * 2.0 ** -24 * adb, f"db at {off}, {pad}")
        assert lf.rel(dw, rdw) < 1e-5 and lf.rel(dx, rdx) < lf.U[dtype] + 1e-5


def test_without_parameters_and_in_leading_axes():
    from paper_2604_10103_b200 import layers
    x, _, b, dy = make(24, 128, F32)
    y, mean, rstd = layers.layer_norm(x.view(2, 3, 4, 128))
    assert y.shape == (2, 3, 4, 128) and mean.shape == (24,)
    assert lf.rel(y.view(24, 128), lf.norm(x, None, None, 1e-6, 0.0, 0)[0]) < 1e-6
    y2, _, _ = layers.layer_norm(x, None, b)
    assert lf.rel(y2, lf.norm(x, None, b, 1e-6, 0.0, 0)[0]) < 1e-6
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd)
    rdx, rdw, rdb, _, _ = lf.norm_backward(dy, x, mean, rstd, None, 0.0, 0)
    assert lf.rel(dx, rdx) < 1e-6 and lf.rel(dw, rdw) < 1e-6 and lf.rel(db, rdb) < 1e-6


def test_gradients_against_differences():
    """L = sum of y r along random directions: central differences of the 64-bit forward, error of the step h^2 L''' / 6 ~ 1e-9."""
    from paper_2604_10103_b200 import layers
    rows, width, group, h = 12, 160, 4, 1e-5
    x, w, b, r = make(rows, width, F32, group)
    _, mean, rstd = layers.layer_norm(x, w, b, weight_offset=1.0, rows_per_group=group)
    dx, dw, db = layers.layer_norm_backward(r, x, mean, rstd, w, weight_offset=1.0, rows_per_group=group)
    gen = torch.Generator().manual_seed(3)
    for grad, which in ((dx, 0), (dw, 1), (db, 2)):
        args = [lf.f64(x), lf.f64(w), lf.f64(b)]
        v = torch.randn(args[which].shape, generator=gen, dtype=torch.float64)
        ends = []
        for s in (1, -1):
            moved = list(args)
            moved[which] = args[which] + s * h * v
            ends.append((lf.norm(*moved, 1e-6, 1.0, group)[0] * lf.f64(r)).sum())
        diff = float(ends[0] - ends[1]) / (2 * h)
        got = float((lf.f64(grad) * v).sum())
        assert abs(got - diff) <= 1e-5 * float((lf.f64(grad) * v).abs().sum()), which


def test_a_row_of_nan_or_infinity_stays_alone():
    from paper_2604_10103_b200 import layers
    for dtype in (BF, F32):
        x, w, b, dy = make(40, 512, dtype)
        ref = layers.layer_norm(x, w, b)
        bad = x.clone()
        bad[7, 3], bad[11, 500] = float("nan"), float("inf")
        got = layers.layer_norm(bad, w, b)
        keep = [i for i in range(40) if i not in (7, 11)]
        assert torch.equal(ref[0][keep], got[0][keep]) and torch.isnan(got[0][7]).all() and torch.isnan(got[0][11]).all()
        dx, dw, db = layers.layer_norm_backward(dy, bad, got[1], got[2], w)
        rx, _, rb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w)
        assert torch.equal(dx[keep], rx[keep]) and torch.equal(db, rb) and torch.isnan(dw).any()


def test_constant_rows_and_large_offsets():
    """A row of one value has variance 0: rstd = 1 / sqrt(eps), xhat 0.  A large common offset costs the mean's bits, not the variance."""
    from paper_2604_10103_b200 import layers
    x = torch.full((3, 320), 7.25, device="cuda")
    y, mean, rstd = layers.layer_norm(x, eps=1e-4)
    assert torch.equal(mean, torch.full_like(mean, 7.25)) and torch.equal(y, torch.zeros_like(y))
    assert torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-6)
    x, _, _, _ = make(8, 640, F32, shift=4096.0)
    y, _, _ = layers.layer_norm(x)
    ry, _, rrstd, xhat, a = lf.norm(x, None, None, 1e-6, 0.0, 0)
    lf.close(y, ry, forward_bound(x, ry, xhat, a, 0.0, rrstd, F32), "y")


def test_no_rows_one_stream_of_its_own_and_a_graph():
    from paper_2604_10103_b200 import layers
    e = torch.empty(0, 64, device="cuda")
    y, mean, rstd = layers.layer_norm(e)
    dx, dw, db = layers.layer_norm_backward(e, e, mean, rstd)
    assert y.shape == (0, 64) and dx.shape == (0, 64) and not dw.any() and not db.any() and dw.shape == (1, 64)
    x, w, b, dy = make(1000, 1536, BF)
    ref = layers.layer_norm(x, w, b)
    refb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = layers.layer_norm(x, w, b)
        gotb = layers.layer_norm_backward(dy, x, got[1], got[2], w)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref + refb, got + gotb))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g1 = layers.layer_norm(x, w, b)
        g2 = layers.layer_norm_backward(dy, x, g1[1], g1[2], w)
    for t in g1 + g2:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref + refb, g1 + g2))


def test_in_place():
    from paper_2604_10103_b200 import binding as hf, layers
    x, w, b, dy = make(50, 768, BF)
    y, mean, rstd = layers.layer_norm(x, w, b)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w)
    s = hf.hf_norm_shape(type=0, param_type=0, width=768, rows=50, x_stride=768, y_stride=768, dx_stride=768, rows_per_group=0, param_stride=768,
                         weight_offset=0.0, eps=1e-6)
    ws = torch.empty(hf.hf_layer_norm_workspace(C.byref(s)), dtype=torch.uint8, device="cuda")
    g, gw, gb = dy.clone(), torch.empty_like(dw), torch.empty_like(db)
    hf.hf_layer_norm_backward(C.byref(s), g, x, mean, rstd, w, g, gw, gb, ws)          # dx over dy
    assert torch.equal(g, dx) and torch.equal(gw, dw) and torch.equal(gb, db)
    g = dy.clone()
    hf.hf_layer_norm_backward(C.byref(s), g, x, mean, rstd, w, None, gw, gb, ws)       # the parameters' gradients alone
    assert torch.equal(gw, dw) and torch.equal(g, dy)
    hf.hf_layer_norm_backward(C.byref(s), dy, x, mean, rstd, w, g, None, None, None)   # dx alone
    assert torch.equal(g, dx)
    z = x.clone()
    hf.hf_layer_norm(C.byref(s), z, w, b, z, None, None)
    assert torch.equal(z, y)
