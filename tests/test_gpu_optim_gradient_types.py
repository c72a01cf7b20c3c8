"""Gradients whose type changes from step to step: the parameters' type and float32 are both taken."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def parameters(dtype=BF, n=3):
    ps = [torch.nn.Parameter(torch.linspace(-1.0, 1.0, 300 + i, device="cuda").to(dtype)) for i in range(n)]
    for p in ps:
        p.grad_dtype = None             # (any type)
        p.grad = torch.linspace(1.0, 2.0, p.numel(), device="cuda").to(dtype)
    return ps


def test_bf16_gradients_and_then_float32_ones():
    from paper_2604_10103_b200 import optim
    a, b = parameters(), parameters()
    one, two = optim.AdamW(a, lr=0.1), optim.AdamW(b, lr=0.1)
    for dtype in (BF, BF, F32, F32, BF):
        for p, q in zip(a, b):
            p.grad, q.grad = p.grad.to(dtype), q.grad.to(F32)           # (the same values)
        one.step()
        two.step()
    assert all(torch.equal(one.state[p]["master"], two.state[q]["master"]) for p, q in zip(a, b))
    a[1].grad = a[1].grad.to(F32)       # of both types in a step
    one.step()
    two.step()
    assert all(torch.equal(one.state[p]["master"], two.state[q]["master"]) for p, q in zip(a, b)) and int(one.state[a[1]]["step"]) == 6
