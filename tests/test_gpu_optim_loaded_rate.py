"""A learning rate that lies on the device stays where it is when a state is loaded: a captured step goes on reading it, and two optimizers never share it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def optimizer(lr, value=1.0, **kw):
    from paper_2604_10103_b200 import optim
    p = torch.nn.Parameter(torch.full((300,), value, device="cuda"))
    p.grad = torch.ones_like(p)
    return optim.AdamW([p], lr=lr, weight_decay=0.0, **kw), p


def rate(value, *shape):
    return torch.full(shape, value, device="cuda")


def test_a_captured_step_follows_the_loaded_rate():
    opt, p = optimizer(rate(0.5))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        opt.step()
    at = opt.param_groups[0]["lr"].data_ptr()
    for saved in (rate(0.125), rate(0.125, 1), torch.tensor(0.125), 0.125):
        other, _ = optimizer(0.25)
        state = other.state_dict()
        state["param_groups"][0]["lr"] = saved
        opt.param_groups[0]["lr"].fill_(0.5)
        opt.load_state_dict(state)
        lr = opt.param_groups[0]["lr"]
        assert lr.data_ptr() == at and float(lr) == 0.125 and lr.shape == ()
        before = p.detach().clone()
        g.replay()
        # (a constant gradient's quotient is 1 in a first step, up to eps and float32)
        assert ((before - p.detach() - 0.125).abs() < 1e-5).all()
        opt.step()
        assert int(opt.state[p]["step"]) == 2


def test_two_optimizers_do_not_share_it():
    a, _ = optimizer(rate(0.5))
    for mine in (rate(0.25), 0.25):
        b, p = optimizer(mine)
        b.load_state_dict(a.state_dict())
        lr = b.param_groups[0]["lr"]
        assert isinstance(lr, torch.Tensor) and float(lr) == 0.5 and lr.data_ptr() != a.param_groups[0]["lr"].data_ptr()
        a.param_groups[0]["lr"].fill_(0.75)
        assert float(lr) == 0.5
        a.param_groups[0]["lr"].fill_(0.5)
        before = p.detach().clone()
        b.step()
        assert ((before - p.detach() - 0.5).abs() < 1e-5).all()


def test_a_state_brought_by_the_host(tmp_path):
    a, _ = optimizer(rate(0.5))
    a.step()
    torch.save(a.state_dict(), tmp_path / "s.pt")
    for mine in (rate(0.25), 0.25):
        b, p = optimizer(mine)
        b.load_state_dict(torch.load(tmp_path / "s.pt", map_location="cpu"))
        assert float(b.param_groups[0]["lr"]) == 0.5
        b.step()
        assert int(b.state[p]["step"]) == 2


def test_a_rate_of_several_elements_is_refused_before_anything_is_changed():
    a, p = optimizer(0.5)
    b, _ = optimizer(0.25)
    b.step()
    state = b.state_dict()
    state["param_groups"][0]["lr"] = rate(0.5, 2)
    with pytest.raises(ValueError, match="lr"):
        a.load_state_dict(state)
    assert int(a.state[p]["step"]) == 0 and a.param_groups[0]["lr"] == 0.5
