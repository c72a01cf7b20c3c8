"""Layer norm's gradients for rows whose mean is many times their spread: the difference from the mean is formed before it is scaled, so the offset costs the
gradients nothing.

xhat is off by its subtraction's and its product's rounding, 2 x 2^-24 of itself, whatever the mean (it is an input).  dw adds `rows` products, each with
one more rounding; dx adds sums over the row, whose terms follow one another in a thread (at most 48) and a tree."""
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype,offset,spread", [(F32, 4096.0, 1.0), (F32, 1e5, 3.0), (BF, 256.0, 4.0), (HALF, 256.0, 1.0)])
@pytest.mark.parametrize("rows,width", [(40, 64), (33, 641), (300, 1536), (9, 12000), (7, 11999)])
def test_gradients(rows, width, dtype, offset, spread):
    from paper_2604_10103_b200 import layers
    g = torch.Generator().manual_seed(width)
    x = (offset + spread * torch.randn(rows, width, generator=g)).to(dtype).cuda()
    w, dy = torch.randn(1, width, generator=g).to(dtype).cuda(), torch.randn(rows, width, generator=g).to(dtype).cuda()
    _, mean, rstd = layers.layer_norm(x, w)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w)
    rdx, rdw, rdb, adw, adb = lf.norm_backward(dy, x, mean, rstd, w, 0.0, 0)
    e = 2.0 ** -24
    lf.close(db, rdb, (rows + 8) * e * adb, "db")
    lf.close(dw, rdw, (rows + 8) * e * adw, "dw")
    r, xhat = lf.f64(rstd)[:, None], ((lf.f64(x) - lf.f64(mean)[:, None]) * lf.f64(rstd)[:, None]).abs()
    gh = (lf.f64(dy) * lf.f64(w)).abs()
    scale = r * (gh + gh.mean(1, keepdim=True) + xhat * (gh * xhat).mean(1, keepdim=True))
    lf.close(dx, rdx, lf.U[dtype] * rdx.abs() + lf.TINY[dtype] + (width / 128 + 64) * e * scale, "dx")
