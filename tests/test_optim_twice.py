"""A parameter that is given twice would be read and written by two parts of a launch at the same time: it is refused, without a device too.  (torch refuses
one that is in two groups, and warns of one that is twice in a group.)"""
import warnings

import pytest
import torch

from paper_2604_10103_b200 import optim


@pytest.mark.parametrize("groups", [lambda p, q: [p, q, p], lambda p, q: [dict(params=[q]), dict(params=[p, p])], lambda p, q: [dict(params=[p]), dict(params=[q, p])]])
def test_the_same_parameter_twice(groups):
    p, q = (torch.nn.Parameter(torch.zeros(4)) for _ in range(2))
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with pytest.raises(ValueError, match="twice|more than one"):
            optim.AdamW(groups(p, q))
