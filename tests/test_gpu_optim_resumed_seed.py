"""A run in 8 bits that is stored and resumed rounds as the one that goes on: the seed is part of the state."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def optimizer(p, seed):
    from paper_2604_10103_b200 import optim
    return optim.AdamW([p], lr=0.1, state_bits=8, seed=seed)


def parameter(value):
    p = torch.nn.Parameter(value.clone())
    p.grad = torch.linspace(-1.0, 1.0, 3000, device="cuda")
    return p


def test_resumed(tmp_path):
    p = parameter(torch.linspace(0.0, 1.0, 3000, device="cuda"))
    a = optimizer(p, 2 ** 32 + 77)
    a.step()
    torch.save(dict(opt=a.state_dict(), p=p.detach()), tmp_path / "s.pt")
    saved = torch.load(tmp_path / "s.pt")
    q = parameter(saved["p"])
    b = optimizer(q, 0)
    b.load_state_dict(saved["opt"])
    assert b.seed == a.seed == 77
    for _ in range(3):
        a.step()
        b.step()
    assert torch.equal(p, q) and all(torch.equal(a.buffers[k].view(torch.uint8), b.buffers[k].view(torch.uint8)) for k in ("m", "v", "scales"))


def test_a_state_without_a_seed_keeps_the_optimizers_own():
    p = parameter(torch.zeros(3000, device="cuda"))
    a = optimizer(p, 5)
    state = a.state_dict()
    state.pop("seed", None)
    b = optimizer(parameter(torch.zeros(3000, device="cuda")), 9)
    b.load_state_dict(state)
    assert b.seed == 9
