"""The gradients' norm over parameters of which some have none, as a step takes them: they are left out."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_missing_gradients_are_left_out():
    from paper_2604_10103_b200 import optim
    ps = [torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (3, 500, 70)]
    ps[0].grad, ps[2].grad = torch.randn(3, device="cuda"), torch.randn(70, device="cuda")
    got = optim.gradient_norm([p.grad for p in ps], 0.5)
    want = optim.gradient_norm([ps[0].grad, ps[2].grad], 0.5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    opt = optim.AdamW(ps, lr=0.1)
    opt.step(grad_factor=got[1])
    assert [int(opt.state[p]["step"]) for p in ps] == [1, 0, 1]
    with pytest.raises(ValueError, match=r"tensors\[2\]"):
        optim.gradient_norm([None, ps[0].grad, torch.zeros(4, device="cuda", dtype=torch.float64)])
