"""A linear layer's backward pass over no rows: sums over nothing are 0, the gradient of a gate without groups too (it has one row, whatever the rows)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def memory_that_is_not_zero():
    """What the allocator hands out next holds sevens."""
    torch.cuda.empty_cache()
    for size in (64, 128, 512, 1024, 8192, 65536):
        for t in [torch.full((size,), 7.0, device="cuda") for _ in range(8)]:
            del t


@pytest.mark.parametrize("gate_shape,ptype", [((128,), BF), ((1, 128), BF), ((128,), F32)])
@pytest.mark.parametrize("act", [None, "silu"])
def test_a_gate_without_groups(gate_shape, ptype, act):
    from paper_2604_10103_b200 import layers
    x, w, dy = torch.empty(0, 64, dtype=BF, device="cuda"), torch.randn(128, 64, device="cuda").to(BF), torch.empty(0, 128, dtype=BF, device="cuda")
    gate = torch.randn(gate_shape, device="cuda").to(ptype)
    y, pre = layers.linear(x, w, act=act, gate=gate, save=True)
    assert y.shape == (0, 128)
    dx, dw, db, dg = layers.linear_backward(dy, x, w, pre, act, gate)
    assert dg.shape == (1, 128) and (dg == 0).all() and (dw == 0).all() and (db == 0).all() and dx.shape == (0, 64)
    dg = layers.linear_backward(dy, x, w, pre, act, gate, dx=False, dweight=False, dbias=False)[3]
    assert (dg == 0).all()
    assert layers.linear_backward(dy, x, w, pre, act, gate[:0].view(0, 128), 5)[3].shape == (0, 128)       # in groups: none of them
    gate.requires_grad_()
    layers.linear(x, w, act=act, gate=gate).sum().backward()
    assert gate.grad.shape == gate_shape and (gate.grad == 0).all()


def test_written_through_the_binding():
    """The memory that the call is given."""
    from paper_2604_10103_b200 import binding as hf, layers
    w, gate, out = torch.zeros(128, 64, dtype=BF, device="cuda"), torch.ones(128, dtype=BF, device="cuda"), torch.full((3, 128), 7.0, device="cuda")
    nothing = torch.empty(0, dtype=BF, device="cuda")
    for group, rows in ((0, [0.0]), (5, [])):
        out.fill_(7.0)
        shape = layers._LINEAR(hf.HF_BF16, hf.HF_BF16, hf.HF_ACT_NONE, 64, 128, 0, 64, 128, 128, group, 128)
        hf.hf_linear_backward(shape, nothing, nothing, w, nothing, gate, None, None, None, out, None)
        assert out[:, 0].tolist() == rows + [7.0] * (3 - len(rows)) and (out == out[:, :1]).all()
