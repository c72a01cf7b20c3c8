"""A step that is refused changes no parameter, whichever of its launches the refusal is about."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, HALF = torch.bfloat16, torch.float32, torch.float16


def parameters(dtype=BF, n=3):
    ps = [torch.nn.Parameter(torch.linspace(-1.0, 1.0, 300 + i, device="cuda").to(dtype)) for i in range(n)]
    for p in ps:
        p.grad_dtype = None             # (any type)
        p.grad = torch.linspace(1.0, 2.0, p.numel(), device="cuda").to(dtype)
    return ps


@pytest.mark.parametrize("dtype,bad", [(BF, HALF), (F32, BF), (F32, HALF), (F32, torch.float64)])
def test_a_gradient_of_a_type_that_is_not_taken(dtype, bad):
    from paper_2604_10103_b200 import optim
    ps = parameters(dtype)
    opt = optim.AdamW(ps, lr=0.1)
    for steps in (0, 1):                # without kept tables, and with them
        before = [p.detach().clone() for p in ps]
        good, ps[2].grad = ps[2].grad, ps[2].grad.to(bad)
        with pytest.raises(ValueError, match="gradient"):
            opt.step()
        assert all(torch.equal(p, q) for p, q in zip(ps, before)) and [int(opt.state[p]["step"]) for p in ps] == [steps] * 3
        ps[2].grad = good
        opt.step()


@pytest.mark.parametrize("kw", [dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(betas=(0.9, float("nan"))), dict(eps=-1.0), dict(eps=float("inf"))])
def test_settings_of_a_later_group_that_are_not_taken(kw):
    from paper_2604_10103_b200 import optim
    ps = parameters(F32)
    opt = optim.AdamW([dict(params=ps[:2]), dict(params=ps[2:])], lr=0.1)
    opt.param_groups[1].update(kw)
    before = [p.detach().clone() for p in ps]
    with pytest.raises(ValueError, match="betas|eps"):
        opt.step()
    assert all(torch.equal(p, q) for p, q in zip(ps, before)) and [int(opt.state[p]["step"]) for p in ps] == [0] * 3
