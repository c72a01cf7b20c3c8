"""Rows of one value: their mean is that value, their variance 0, however many rows there are (few rows and many take different kernels).  The sums are
exact here: 8 bits of a value and 12 of a width fit in float32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,width", [(5, 1455), (6000, 1455), (6000, 1456), (6000, 96), (6000, 97), (6000, 1537), (2000, 3001)])
def test_forward(rows, width, dtype):
    from paper_2604_10103_b200 import layers
    values = torch.tensor([1.0, 3.0, 7.25, 100.0, -201.0, 255.0, 0.0], device="cuda")
    x = values[torch.arange(rows, device="cuda") % 7][:, None].expand(rows, width).to(dtype).contiguous()
    y, mean, rstd = layers.layer_norm(x, eps=1e-4)
    assert torch.equal(mean, x[:, 0].float()) and not y.any()
    assert torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-6)


@pytest.mark.parametrize("rows,width", [(5, 1455), (6000, 97), (6000, 1537)])
def test_the_mean_of_a_row_with_an_infinity(rows, width):
    from paper_2604_10103_b200 import layers
    x = torch.ones(rows, width, device="cuda").bfloat16()
    x[1, 3], x[3, width - 1], x[4, 0] = float("inf"), -float("inf"), float("nan")
    y, mean, rstd = layers.layer_norm(x)
    assert mean[:4].tolist() == [1.0, float("inf"), 1.0, -float("inf")] and torch.isnan(mean[4]) and (mean[5:] == 1.0).all()
    assert torch.isnan(y[[1, 3, 4]]).all() and torch.isnan(rstd[[1, 3, 4]]).all() and not y[5:].any()
