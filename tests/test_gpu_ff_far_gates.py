"""Gates as far out as bfloat16 goes: the activation is 0 or the gate, its slope 0 or 1, and nothing on the way (a square of the gate) overflows into
either."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M", [3, 140])
def test_slopes(M, act):
    from paper_2604_10103_b200 import layers
    n = 64
    far = torch.tensor([20.0, -20.0, 1e4, -1e4, 1e18, -1e18, 2e19, -2e19, 1e25, -1e25, 3e38, -3e38]).bfloat16()
    gate = far[torch.arange(M * n) % len(far)].view(M, n).cuda()
    up = torch.ones(M, n).bfloat16().cuda()
    eye = torch.eye(n).bfloat16().cuda()
    x, dy = torch.zeros(M, n).bfloat16().cuda(), torch.zeros(M, n).bfloat16().cuda()
    g = torch.Generator().manual_seed(1)
    dy.copy_(torch.rand(M, n, generator=g) - 0.5)               # (du = dy act(gate) stays finite)
    # wg and wd the identity, wu 0: dh = dy, dx = dg
    none = torch.zeros_like(eye)
    dx = layers.gated_ff_backward(dy, x, eye, none, eye, gate, up, act=act)[0]
    # dx = dg = dy act'(gate); what is left of the slope at -20 is 2e-9 x 20
    want = torch.where(gate > 0, dy, torch.zeros_like(dy))
    assert torch.isfinite(dx).all() and (dx.float() - want.float()).abs().max() < 1e-6
    # the forward pass at the same gates
    y, got, _ = layers.gated_ff(torch.eye(n).bfloat16().cuda(), torch.diag(far[torch.arange(n) % len(far)]).cuda(), torch.ones_like(eye), eye, act=act, save=True)
    d = torch.diag(got)
    assert torch.equal(d, far[torch.arange(n) % len(far)].cuda())
    want = torch.where(d > 0, d, torch.zeros_like(d)).float()
    assert torch.isfinite(y).all() and ((torch.diag(y).float() - want).abs() <= 2.0 ** -8 * want + 1e-6).all()
