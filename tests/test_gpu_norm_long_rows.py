"""Layer norm's backward pass around the widths where rows of floats get too long for the rings in shared memory, on rows that start on 16 bytes and
on rows that do not, against the definition in 64 bits."""
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("width", [11604, 11605, 11608, 11612, 12001, 12288, 12289, 14337])
def test_backward(width, off):
    from paper_2604_10103_b200 import binding as hf, layers
    rows = 5
    g = torch.Generator().manual_seed(width)
    x, dy, w = torch.randn(rows, width, generator=g), torch.randn(rows, width, generator=g), torch.randn(1, width, generator=g)

    def put(t):
        v = torch.zeros(t.numel() + off, device="cuda")[off:].view(t.shape)
        v.copy_(t)
        return v
    x, dy, w = put(x), put(dy), put(w)
    _, mean, rstd = layers.layer_norm(x, w)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w)
    rdx, rdw, rdb, adw, adb = lf.norm_backward(dy, x, mean, rstd, w, 0.0, 0)
    # five rows' sums in at most five steps and an exact product's rounding each; xhat is off by 2^-22 of |x| rstd + |mean| rstd at most (both near 1 here)
    lf.close(db, rdb, 8 * 2.0 ** -24 * adb, "db")
    lf.close(dw, rdw, 8 * 2.0 ** -24 * adw + 4 * 2.0 ** -24 * adb * (1 + lf.f64(mean).abs().max()), "dw")
    # dx: sums of `width` terms over at least 256 threads, each step within 2^-24 of the absolute terms
    n = (width / 256 + 40) * 2.0 ** -24
    gh, xhat = (lf.f64(dy) * lf.f64(w)).abs(), ((lf.f64(x) - lf.f64(mean)[:, None]) * lf.f64(rstd)[:, None]).abs()
    scale = lf.f64(rstd)[:, None] * (gh + gh.mean(1, keepdim=True) + (1 + xhat) * (1 + (gh * xhat).mean(1, keepdim=True)))
    lf.close(dx, rdx, n * scale, "dx")
    assert hf.hf_layers_status() == (0, 0)
