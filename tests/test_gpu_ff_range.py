"""The gated feed-forward in float16 at both ends of the type's range: what lies between the products is held in it."""
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
HALF, BF = torch.float16, torch.bfloat16


def aimed(M, n, dtype, gate, up):
    """x one hot, weights diagonal: g = gate, u = up on every diagonal element, y = their act(g) u, with nothing else in the sums."""
    x = torch.zeros(M, n)
    x[torch.arange(M), torch.arange(M) % n] = 1.0
    eye = torch.eye(n)
    return [t.to(dtype).cuda() for t in (x, gate * eye, up * eye, eye)]


@pytest.mark.parametrize("M", [1, 16, 17, 150])
def test_the_largest_products(M):
    """255 x 255 = 65025 and 255.875 x 256 = 65504 are held; 256 x 256 is not, in float16, and stays in its own row."""
    from paper_2604_10103_b200 import layers
    n = 64
    for gate, up in ((255.0, 255.0), (255.875, 256.0), (255.0, -255.0)):
        y = layers.gated_ff(*aimed(M, n, HALF, gate, up))
        at = (torch.arange(M), torch.arange(M) % n)
        want = torch.zeros(M, n, dtype=torch.float64)
        want[at] = gate * up
        # gate up needs more bits than the type has: one rounding of h (y is h)
        lf.close(y, want, lf.U[HALF] * want.abs(), f"{gate} x {up}")
    x, wg, wu, wd = aimed(M, n, HALF, 1.0, 1.0)
    x[M // 2] *= 256.0
    y = layers.gated_ff(x, wg, wu, wd)
    assert not torch.isfinite(y[M // 2]).all()
    others = [i for i in range(M) if i != M // 2]
    x[M // 2] /= 256.0
    assert torch.isfinite(y[others]).all() and torch.equal(y[others], layers.gated_ff(x, wg, wu, wd)[others])
    # bfloat16 holds it
    y = layers.gated_ff(*aimed(M, n, BF, 256.0, 256.0))
    assert float(y.max()) == 65536.0 and torch.isfinite(y).all()


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M", [9, 200])
def test_gradients_below_the_smallest_normal_number(M, act):
    """dy scaled by 2^-k: each of dg, du is off by U of itself or by half the spacing of float16's subnormals, 2^-25; dx carries |W| of that and
    its own rounding.  With a dy of ordinary size the same gradient keeps its relative accuracy."""
    from paper_2604_10103_b200 import layers
    K, N, O = 64, 128, 64
    g = torch.Generator().manual_seed(M)
    x, dy = (torch.randn(M, n, generator=g).to(HALF).cuda() for n in (K, O))
    wg, wu, wd = ((torch.randn(*s, generator=g) / s[1] ** 0.5).to(HALF).cuda() for s in ((N, K), (N, K), (O, N)))
    _, gate, up = layers.gated_ff(x, wg, wu, wd, act=act, save=True)
    for k in (0, 6, 10):
        small = dy * 2.0 ** -k
        dx = layers.gated_ff_backward(small, x, wg, wu, wd, gate, up, act=act)[0]
        rdx, _, _, _, rdg, rdu, _ = lf.ff_backward(small, x, wg, wu, wd, gate, up, act)
        u, half = lf.U[HALF], 2.0 ** -25
        e = (u + 64 * 2.0 ** -24) * (rdg.abs() @ lf.f64(wg).abs() + rdu.abs() @ lf.f64(wu).abs()) + half * (lf.f64(wg).abs().sum(0) + lf.f64(wu).abs().sum(0))
        # float32 error of dh (64 terms) in dg and du: 2^-24 x 64 of the absolute terms, with factors up to 1.2 |u| and |g| + 0.2
        adh = lf.f64(small).abs() @ lf.f64(wd).abs()
        e = e + 64 * 2.0 ** -24 * ((adh * 1.2 * lf.f64(up).abs()) @ lf.f64(wg).abs() + (adh * (lf.f64(gate).abs() + 0.2)) @ lf.f64(wu).abs())
        lf.close(dx, rdx, (1 + u) * e + u * rdx.abs() + half, f"dx at 2^-{k}")
    assert lf.rel(layers.gated_ff_backward(dy, x, wg, wu, wd, gate, up, act=act)[0], lf.ff_backward(dy, x, wg, wu, wd, gate, up, act)[0]) < lf.U[HALF]
