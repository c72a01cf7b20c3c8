"""Gradients through torch's graph over no rows, as a sum over the output gives them: an expanded tensor of no elements, all of whose strides are 0 (torch
counts it as contiguous).  The operators' own gradients are zeros, or have no elements."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def leaf(*shape, dtype=BF):
    return torch.ones(shape, dtype=dtype, device="cuda").requires_grad_()


def grads_of(outs, leaves):
    total = sum(o.sum() for o in (outs if isinstance(outs, tuple) else (outs,)))
    grads = torch.autograd.grad(total, leaves)
    assert all(g.shape == t.shape and (g == 0).all() for g, t in zip(grads, leaves))


@pytest.mark.parametrize("shape", [(0, 64), (0, 3, 64), (2, 0, 64)])
def test_rows(shape):
    from paper_2604_10103_b200 import layers
    x, w, b = leaf(*shape), leaf(64), leaf(64)
    grads_of(layers.layer_norm(x, w, b)[0], (x, w, b))
    m, bias, res = leaf(128, 64), leaf(128), leaf(*shape[:-1], 128)
    grads_of(layers.linear(x, m, bias, act="silu", residual=res), (x, m, bias, res))
    grads_of(layers.linear(x, m), (x, m))
    up, down = leaf(128, 64), leaf(64, 128)
    grads_of(layers.gated_ff(x, m, up, down), (x, m, up, down))


def tables():
    entries = 9 * 12 + 5 * 10 + 6 * 10
    return torch.ones(entries, device="cuda"), torch.zeros(entries, device="cuda"), (9, 5, 6), (12, 10, 10)


@pytest.mark.parametrize("B,T", [(1, 0), (2, 0), (0, 3)])
def test_heads(B, T):
    from paper_2604_10103_b200 import layers
    pos = torch.zeros(T, 3, dtype=torch.int32, device="cuda")
    x = leaf(B, T, 4, 64)
    grads_of(layers.rope_axes(x, pos, tables()), (x,))
    qkv, qw, kw = leaf(B, T, 8 * 64), leaf(64), leaf(64)
    grads_of(layers.split_heads_rope(qkv, 4, 2, pos, tables()), (qkv,))
    grads_of(layers.split_heads_norm_rope(qkv, 4, 2, qw, kw, pos, tables()), (qkv, qw, kw))
    wide = leaf(4 * 64), leaf(2 * 64)
    grads_of(layers.split_heads_norm_rope(qkv, 4, 2, *wide, pos, tables(), over="width"), (qkv, *wide))
