"""Thread blocks of many warps with key heads whose teams leave some of them over, norms over the width: 16 warps with teams of three, five, six, seven and nine."""
import pytest
import torch

from tests.test_gpu_heads_norm_rope import check, no_position_outside  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,KV,d", [(128, 24, 128), (128, 40, 128), (128, 44, 128), (128, 52, 128), (64, 36, 256), (250, 48, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_teams_that_leave_warps_over(H, KV, d, dtype):
    check(1, 23, H, KV, d, dtype, "width", "adjacent", (8, 4, 4))
