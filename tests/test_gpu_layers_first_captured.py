"""Calls without a context may be captured once one call of the kind has been made on the device, whatever its size: kernels are chosen by size, and
those that a larger call takes have not run before the capture."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import torch
from paper_2604_10103_b200 import binding as hf, layers, rope

def t(*s, dtype=torch.bfloat16):
    return torch.randn(*s, device="cuda").to(dtype)

extents, pairs = (6, 5, 4), (12, 10, 10)
tab = tuple(torch.from_numpy(a).cuda() for a in rope.axis_tables(extents, pairs)) + (extents, pairs)

def ff(M, K, N, dtype):
    x, wg, wu, wd, dy = t(M, K, dtype=dtype), t(N, K, dtype=dtype), t(N, K, dtype=dtype), t(K, N, dtype=dtype), t(M, K, dtype=dtype)
    def calls():
        y, g, u = layers.gated_ff(x, wg, wu, wd, save=True)
        return (y, g, u) + layers.gated_ff_backward(dy, x, wg, wu, wd, g, u)
    return calls

def norm(R, W, dtype):
    x, w, dy = t(R, W, dtype=dtype), t(1, W, dtype=dtype), t(R, W, dtype=dtype)
    def calls():
        y, m, r = layers.layer_norm(x, w, w)
        return (y, m, r) + layers.layer_norm_backward(dy, x, m, r, w)
    return calls

def turn(T, dtype, pairing):
    pos = torch.zeros(T, 3, dtype=torch.int32, device="cuda")
    x = t(1, T, 6 * 64, dtype=dtype)
    return lambda: layers.split_heads_rope(x, 2, 2, pos, tab, pairing=pairing)

B, H, F = torch.bfloat16, torch.float16, torch.float32
first = [ff(2, 64, 64, B), norm(2, 64, B), turn(3, B, "adjacent")]
then = [ff(17, 64, 128, B), ff(77, 512, 1024, H), ff(300, 512, 1024, B), ff(1000, 1536, 1024, B), ff(2500, 512, 1024, H), ff(3, 64, 64, H),
        norm(5, 65, F), norm(3000, 1536, B), norm(3000, 1535, H), norm(400, 4096, F), norm(40, 16383, F), norm(40, 12001, F), turn(900, H, "halves"), turn(77, F, "adjacent")]
for f in first:
    f()
torch.cuda.synchronize()
for f in then:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = f()
    graph.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in got]
    ref = f()
    assert all(torch.equal(p, q) for p, q in zip(got, ref))
    graph.reset()
assert hf.hf_layers_status() == (0, 0)
print("captured")
"""


@pytest.mark.parametrize("lazy", ["LAZY", "EAGER"])
def test_larger_calls(lazy):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300, env=dict(os.environ, CUDA_MODULE_LOADING=lazy))
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
