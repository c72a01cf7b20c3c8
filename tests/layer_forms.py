"""Plain 64-bit forms of the block operators (layer norm, rotary positions, gated feed-forward) for the tests, and the bounds that the
tests derive from the kernels' roundings.

U[type]: half a unit in the last place, relative.  A result computed in float32 and rounded once is off by U |result| plus the float32
error, which is bounded by n 2^-24 times the sum of the absolute terms for a sum of n terms."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -24, torch.float32: 1e-38}      # (the type's subnormal spacing)


def f64(t):
    return None if t is None else t.detach().double().cpu()


def groups_of(rows, rows_per_group):
    return torch.arange(rows) // rows_per_group if rows_per_group else torch.zeros(rows, dtype=torch.long)


def norm(x, w, b, eps, offset, rows_per_group):
    x, w, b = f64(x), f64(w), f64(b)
    of = groups_of(x.shape[0], rows_per_group)
    mean = x.mean(1)
    rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    a = torch.ones_like(xhat) if w is None else (w + offset).reshape(-1, x.shape[1])[of]
    return xhat * a + (0.0 if b is None else b.reshape(-1, x.shape[1])[of]), mean, rstd, xhat, a


def norm_backward(dy, x, mean, rstd, w, offset, rows_per_group):
    dy, x, mean, rstd, w = f64(dy), f64(x), f64(mean)[:, None], f64(rstd)[:, None], f64(w)
    of = groups_of(x.shape[0], rows_per_group)
    xhat = (x - mean) * rstd
    a = torch.ones_like(x) if w is None else (w + offset).reshape(-1, x.shape[1])[of]
    gh = dy * a
    dx = rstd * (gh - gh.mean(1, keepdim=True) - xhat * (gh * xhat).mean(1, keepdim=True))
    groups = -(-x.shape[0] // rows_per_group) if rows_per_group else 1

    def total(v):
        return torch.zeros(groups, x.shape[1], dtype=torch.float64).index_add_(0, of, v)
    return dx, total(dy * xhat), total(dy), total((dy * xhat).abs()), total(dy.abs())


def rope(x, pos, cos, sin, extents, pairs, halves, inverse):
    """x [B, T, H, d]; pos [T, A] or [B, T, A]; a loop over axes and pairs."""
    x, cos, sin, pos = f64(x), f64(cos), f64(sin), pos.cpu().long()
    if pos.dim() == 2:
        pos = pos[None]
    pos = pos.expand(x.shape[0], -1, -1)
    y, P, p, start = x.clone(), sum(pairs), 0, 0
    for a, (e, n) in enumerate(zip(extents, pairs)):
        for j in range(n):
            at = start + pos[..., a] * n + j
            c, s = cos[at][..., None], (-sin if inverse else sin)[at][..., None]
            i0, i1 = (p, P + p) if halves else (2 * p, 2 * p + 1)
            y[..., i0] = x[..., i0] * c - x[..., i1] * s
            y[..., i1] = x[..., i0] * s + x[..., i1] * c
            p += 1
        start += e * n
    return y


def act(g, name):
    if name == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))


def ff(x, wg, wu, wd, name):
    x, wg, wu, wd = f64(x), f64(wg), f64(wu), f64(wd)
    g, u = x @ wg.t(), x @ wu.t()
    h = act(g, name) * u
    return h @ wd.t(), g, u, h


def ff_backward(dy, x, wg, wu, wd, gate, up, name):
    """At the saved gate and up, by differentiating act(gate) up."""
    dy, x, wg, wu, wd = f64(dy), f64(x), f64(wg), f64(wu), f64(wd)
    g, u = f64(gate).requires_grad_(), f64(up).requires_grad_()
    h = act(g, name) * u
    dg, du = torch.autograd.grad(h, (g, u), dy @ wd)
    return dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h.detach(), dg, du, h.detach()


def close(got, ref, bound, what):
    """Every element within its bound; NaN and infinities where the reference has them."""
    got, bound = f64(got), torch.as_tensor(bound, dtype=torch.float64).expand_as(ref)
    assert got.shape == ref.shape, f"{what}: {tuple(got.shape)} instead of {tuple(ref.shape)}"
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: finite in other places"
    over = ((got - ref).abs() - bound)[fine]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: over its bound by {over.max():.3e} of {bound[fine][over.argmax()]:.3e}"


def rel(got, ref):
    got = f64(got)
    n = ref.norm()
    return float((got - ref).norm() / n) if n else float(got.norm())
