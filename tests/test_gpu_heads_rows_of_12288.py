"""Norms of q and k over the width, backward, where a row of the weight and the kernel's own shared memory are together just above what a launch has
without being asked for (48 KB): 12225 to 12288 features.  Larger rows ask for more, so these come first in a process of their own."""
import subprocess
import sys

import pytest

from tests.conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,KV,d,pairs", [(96, 8, 128, (22, 21, 21)), (48, 4, 256, (44, 42, 42)), (192, 3, 64, (12, 10, 10)), (128, 2, 96, (16, 16, 16))])
def test_first_in_a_process(H, KV, d, pairs):
    text = f"""
import torch
from tests.test_gpu_heads_norm_rope import check
for dtype in (torch.bfloat16, torch.float32):
    check(1, 5, {H}, {KV}, {d}, dtype, "width", "adjacent", {pairs})
check(2, 3, {H}, {KV}, {d}, torch.float16, "width", "halves", {pairs})
from paper_2604_10103_b200 import binding as hf
assert hf.hf_layers_status() == (0, 0)
"""
    done = subprocess.run([sys.executable, "-c", text], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stderr[-2000:]
