"""A learning rate that is a tensor is read by the kernel where it lies: one that is not a float32 element on the device is refused, subclasses of a tensor
(a Parameter) among them.  Without a device: the settings alone."""
import pytest
import torch

from paper_2604_10103_b200 import optim


class Other(torch.Tensor):
    pass


def settings(*rates):
    o = optim.AdamW.__new__(optim.AdamW)
    o.param_groups = [dict(lr=lr, weight_decay=0.0, betas=(0.9, 0.99), eps=1e-8, params=[]) for lr in rates]
    o._device = 0
    return o._settings()


@pytest.mark.parametrize("kind", [torch.Tensor, torch.nn.Parameter, Other])
def test_a_tensor_that_the_kernel_cannot_read(kind):
    made = {torch.Tensor: lambda t: t, torch.nn.Parameter: torch.nn.Parameter, Other: lambda t: t.as_subclass(Other)}[kind]
    for bad, text in ((torch.tensor(0.1), "not on the current CUDA device"), (torch.tensor(0.1, dtype=torch.float64), "float32"), (torch.ones(2), "one element")):
        assert type(made(bad)) is kind
        for rates in ([made(bad)], [0.1, made(bad)], [made(bad), 0.1]):
            with pytest.raises(ValueError, match=text):
                settings(*rates)


def test_numbers():
    assert settings(0.1, 1) == [(0.1, 0.0, (0.9, 0.99), 1e-8), (1, 0.0, (0.9, 0.99), 1e-8)]
