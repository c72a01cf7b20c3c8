"""Settings that are changed in place take effect in the next step, whatever object holds them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def optimizer(**kw):
    from paper_2604_10103_b200 import optim
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    p.grad = torch.full_like(p, 2.0)
    return optim.AdamW([p], **dict(dict(lr=0.5, eps=0.0, weight_decay=0.0), **kw)), p


def test_betas_of_a_list():
    opt, p = optimizer(betas=[0.5, 0.5])
    opt.step()
    opt.step()                          # (the second goes by the kept tables)
    assert (opt.state[p]["m"] == 1.5).all()
    opt.param_groups[0]["betas"][0] = 0.75
    opt.step()
    assert (opt.state[p]["m"] == 0.75 * 1.5 + 0.25 * 2.0).all()


def test_numbers_that_are_arrays():
    import numpy as np
    lr, decay = np.array(0.5), torch.tensor(0.0)
    opt, p = optimizer(lr=lr, weight_decay=decay)
    opt.step()
    opt.step()
    assert ((p.detach() - 0.0).abs() < 1e-5).all()      # (a constant gradient's quotient is 1)
    lr[()] = 0.25
    opt.step()
    assert ((p.detach() + 0.25).abs() < 1e-5).all()
    decay.fill_(4.0)                    # p - lr (1 + 4 p)
    opt.step()
    assert ((p.detach() - (-0.25 - 0.25 * (1.0 - 1.0))).abs() < 1e-5).all()
