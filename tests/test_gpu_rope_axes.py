"""Rotary positions with several axes against a loop over axes and pairs in 64 bits."""
import numpy as np
import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def no_wait_ran_out():
    """A bounded wait that runs out may leave right numbers behind: the status word tells."""
    yield
    from paper_2604_10103_b200 import binding as hf
    assert hf.hf_layers_status() == (0, 0)


BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


def tables(extents, pairs):
    from paper_2604_10103_b200 import rope
    cos, sin = rope.axis_tables(extents, pairs)
    return torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), extents, pairs


def positions(B, T, extents, seed=0, shared=True):
    g = torch.Generator().manual_seed(seed + T)
    cols = [torch.randint(0, e, (1 if shared else B, T), generator=g) for e in extents]
    p = torch.stack(cols, dim=-1).to(torch.int32).cuda()
    return p[0].contiguous() if shared else p


def bound(x, ref, dtype):
    """Two products and a sum, each within 2^-24 of |x0| + |x1|, then one rounding."""
    m = lf.f64(x).abs()
    m = m + m.amax(-1, keepdim=True)
    return lf.U[dtype] * ref.abs() + lf.TINY[dtype] + 3 * 2.0 ** -24 * m


CASES = [  # B, T, H, d, pairs, extents
    (1, 1, 1, 2, (1,), (4,)),
    (1, 5, 2, 64, (12, 10, 10), (9, 5, 7)),
    (2, 33, 3, 128, (22, 21, 21), (30, 8, 11)),
    (1, 7, 5, 96, (16, 8, 8), (8, 8, 8)),            # 32 features behind the rotated ones
    (1, 7, 5, 96, (8, 16), (8, 8)),                  # two axes, 48 features behind them
    (2, 19, 2, 6, (1, 1, 1), (3, 3, 3)),             # less than a 16-byte piece
    (1, 9, 3, 20, (2, 3, 1, 4), (3, 4, 5, 6)),       # four axes
    (3, 4, 1, 80, (0, 24, 16), (1, 6, 6)),           # an axis without pairs
    (1, 300, 12, 128, (22, 21, 21), (21, 30, 52)),
]


@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("B,T,H,d,pairs,extents", CASES)
def test_against_the_definition(B, T, H, d, pairs, extents, pairing, dtype):
    from paper_2604_10103_b200 import layers
    g = torch.Generator().manual_seed(T * d)
    x = torch.randn(B, T, H, d, generator=g).to(dtype).cuda()
    tab = tables(extents, pairs)
    for shared in (True, False):
        pos = positions(B, T, extents, shared=shared)
        for inverse in (False, True):
            ref = lf.rope(x, pos, tab[0], tab[1], extents, pairs, pairing == "halves", inverse)
            got = layers.rope_axes(x, pos, tab, pairing=pairing, inverse=inverse)
            lf.close(got, ref, bound(x, ref, dtype), f"{pairing} inverse={inverse}")
            tail = 2 * sum(pairs)
            assert torch.equal(got[..., tail:], x[..., tail:])
            # other strides give the same bits: heads first, and one element off every 16-byte boundary
            heads_first = torch.empty(B, H, T, d, dtype=dtype, device="cuda").transpose(1, 2)
            assert torch.equal(layers.rope_axes(x, pos, tab, out=heads_first, pairing=pairing, inverse=inverse), got)
            odd = torch.zeros(B * T * H * (d + 1) + 1, dtype=dtype, device="cuda")[1:].view(B, T, H, d + 1)[..., :d]
            odd.copy_(x)
            assert torch.equal(layers.rope_axes(odd, pos, tab, pairing=pairing, inverse=inverse), got)
            assert torch.equal(layers.rope_axes(odd, pos, tab, out=odd, pairing=pairing, inverse=inverse), got)
    same = x.clone()
    layers.rope_axes(same, pos, tab, out=same, pairing=pairing, inverse=True)
    assert torch.equal(same, got)


@pytest.mark.parametrize("B,T,H,KV,d,pairing", [(1, 64, 2, 2, 64, "adjacent"), (2, 77, 12, 3, 128, "adjacent"), (1, 1, 12, 12, 128, "adjacent"),
                                                (1, 130, 8, 2, 64, "halves"), (2, 1560, 4, 1, 96, "adjacent")])
def test_fused_projection_to_heads_and_back(B, T, H, KV, d, pairing):
    from paper_2604_10103_b200 import layers
    n = d // 2
    pairs, extents = (n - 2 * (n // 3), n // 3, n // 3), (40, 30, 52)
    if pairing == "halves":
        pairs = (n - 16, 8, 8)
    tab, pos = tables(extents, pairs), positions(B, T, extents)
    g = torch.Generator().manual_seed(5)
    W = (H + 2 * KV) * d
    rows = torch.randn(B, T, W + 16, generator=g).to(BF).cuda()[..., 8:8 + W]
    q, k, v = layers.split_heads_rope(rows, H, KV, pos, tab, pairing=pairing)
    x = rows.unflatten(2, (H + 2 * KV, d))
    ref = lf.rope(x[:, :, :H + KV], pos, tab[0], tab[1], extents, pairs, pairing == "halves", False)
    got = torch.cat([q, k], dim=1).transpose(1, 2)
    lf.close(got, ref, bound(x[:, :, :H + KV], ref, BF), "q, k")
    assert torch.equal(v, x[:, :, H + KV:].transpose(1, 2)) and q.is_contiguous() and v.is_contiguous()
    dq, dk, dv = (torch.randn(t.shape, generator=g).to(BF).cuda() for t in (q, k, v))
    back = layers.split_heads_rope_backward(dq, dk, dv, pos, tab, pairing=pairing)
    d_in = torch.cat([dq, dk], dim=1).transpose(1, 2)
    ref = lf.rope(d_in, pos, tab[0], tab[1], extents, pairs, pairing == "halves", True)
    b4 = back.view(B, T, H + 2 * KV, d)
    lf.close(b4[:, :, :H + KV], ref, bound(d_in, ref, BF), "back")
    assert torch.equal(b4[:, :, H + KV:], dv.transpose(1, 2))
    # the backward pass is the transposed map: <R x, g> = <x, R' g>, here in 64 bits
    a = (lf.rope(x, pos, tab[0], tab[1], extents, pairs, pairing == "halves", False) * lf.f64(x.flip(1))).sum()
    b = (lf.f64(x) * lf.rope(x.flip(1), pos, tab[0], tab[1], extents, pairs, pairing == "halves", True)).sum()
    assert abs(float(a - b)) <= 1e-9 * float(lf.f64(x).square().sum())


def test_tables_are_the_angles_of_the_positions():
    from paper_2604_10103_b200 import rope
    cos, sin = rope.axis_tables((5, 3), (4, 2), base=100.0)
    c2, s2 = rope.angle_tables(np.array([[4, 2], [1, 0]]), (4, 2), base=100.0)
    for row, (t, y) in enumerate([(4, 2), (1, 0)]):
        at = [t * 4 + j for j in range(4)] + [20 + y * 2 + j for j in range(2)]
        assert np.array_equal(cos[at], c2[row]) and np.array_equal(sin[at], s2[row])


def test_a_position_outside_its_table_is_reported_and_taken_as_zero():
    from paper_2604_10103_b200 import binding as hf, layers
    extents, pairs = (6, 5), (8, 8)
    tab, pos = tables(extents, pairs), positions(1, 10, extents)
    x = torch.randn(1, 10, 2, 32, device="cuda")
    good = pos.clone()
    good[3, 0], good[7, 1] = 0, 0
    ref = layers.rope_axes(x, good, tab)
    assert hf.hf_layers_status() == (0, 0)
    for bad in (6, -1, 2 ** 31 - 1, -2 ** 31):
        p = good.clone()
        p[3, 0] = bad
        assert torch.equal(layers.rope_axes(x, p, tab), ref)
        with pytest.raises(hf.HFError, match="HF_ERR_INVALID_ARG.*token 3"):
            hf.hf_layers_status()
        assert hf.hf_layers_status() == (0, 0)


def test_infinities_behind_the_rotated_features_are_copied():
    from paper_2604_10103_b200 import layers
    tab, pos = tables((4,), (8,)), torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    x = torch.randn(1, 3, 2, 64, device="cuda").to(BF)
    x[..., 20], x[..., 40], x[..., 63] = float("inf"), float("nan"), -float("inf")
    for pairing in ("adjacent", "halves"):
        y = layers.rope_axes(x, pos, tab, pairing=pairing)
        assert torch.equal(torch.nan_to_num(y[..., 16:], 3.0), torch.nan_to_num(x[..., 16:], 3.0)) and torch.isfinite(y[..., :16]).all()


def test_no_tokens_another_stream_and_a_graph():
    from paper_2604_10103_b200 import layers
    extents, pairs = (6, 5, 4), (12, 10, 10)
    tab = tables(extents, pairs)
    q, k, v = layers.split_heads_rope(torch.empty(1, 0, 6 * 64, device="cuda"), 2, 2, positions(1, 0, extents), tab)
    assert q.shape == (1, 2, 0, 64)
    pos, x = positions(1, 500, extents), torch.randn(1, 500, 6 * 64, device="cuda").to(BF)
    ref = layers.split_heads_rope(x, 2, 2, pos, tab)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = layers.split_heads_rope(x, 2, 2, pos, tab)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layers.split_heads_rope(x, 2, 2, pos, tab)
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
