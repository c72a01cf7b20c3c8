"""Missing gradients are left out of the gradients' norm; where there are no others it is refused, as no tensors are.  No device."""
import pytest
import torch

from paper_2604_10103_b200 import optim


def test_missing_gradients_alone():
    for some in ([None], [None, None]):
        with pytest.raises(ValueError, match="no tensors"):
            optim.gradient_norm(some)
    with pytest.raises(ValueError, match=r"tensors\[1\] is on cpu"):
        optim.gradient_norm([None, torch.zeros(3)])
