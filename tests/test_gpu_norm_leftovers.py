"""Layer norm on multiprocessors whose shared memory an earlier call has left full of NaN: nothing of it reaches a result."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("width", [5, 255, 1027, 1455])
def test_odd_widths(width, dtype):
    """The call before fills its sums over rows, which end in shared memory, with NaN on every multiprocessor; a kernel's shared memory is not
    cleared before the next one starts."""
    from paper_2604_10103_b200 import layers
    g = torch.Generator().manual_seed(width)
    rows = 6000
    x, dy = (torch.randn(rows, width, generator=g).to(dtype).cuda() for _ in range(2))
    w, b = (torch.randn(1, width, generator=g).to(dtype).cuda() for _ in range(2))
    nan = torch.full((rows, width + 1), float("nan"), dtype=dtype, device="cuda")
    ref = layers.layer_norm(x, w, b)
    refb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w)
    torch.cuda.synchronize()
    for _ in range(3):
        layers.layer_norm_backward(nan, nan, nan[:, 0].float().contiguous(), nan[:, 0].float().contiguous())
        got = layers.layer_norm(x, w, b)
        layers.layer_norm_backward(nan, nan, nan[:, 0].float().contiguous(), nan[:, 0].float().contiguous())
        gotb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w)
        assert all(torch.isfinite(t).all() and torch.equal(t, r) for t, r in zip(got + gotb, ref + refb))
