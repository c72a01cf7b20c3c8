"""What linear layers, and norms of q and k with the rotation, refuse before any device call: these run without a device."""
import ctypes as C
import re
import types

import pytest
import torch

from paper_2604_10103_b200 import binding as hf, block as bl, build as hfbuild, inputs as gen, layers
from tests.test_abi import ROOT

INVALID, SHAPE, UNSUPPORTED = 1, 2, 4
P = 0x10000            # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    hfbuild.build()
    return hf.lib()


@pytest.mark.parametrize("name", ["hf_linear_shape", "hf_heads_shape", "hf_heads_tensor"])
def test_structs_match_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(f"{ROOT}/include/hf.h").read(), flags=re.S)
    body = re.findall(r"typedef struct \{([^}]*)\} " + name + ";", text)[0]
    kinds = {"int": C.c_int, "int64_t": C.c_int64, "float": C.c_float, "void*": C.c_void_p}
    want = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        ty, names = re.match(r"(\w+\*?)\s+(.*)", decl, re.S).groups()
        for n in names.split(","):
            m = re.match(r"(\w+)(?:\[(\d+)\])?$", n.strip())
            want.append((m.group(1), kinds[ty] * int(m.group(2)) if m.group(2) else kinds[ty]))
    assert want == list(getattr(hf, name)._fields_)


def linear(**kw):
    return hf.hf_linear_shape(**dict(dict(type=0, param_type=0, act=2, width=64, out_width=128, rows=40, x_stride=64, y_stride=128, residual_stride=128,
                                          rows_per_group=10, gate_stride=128), **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(type=2), UNSUPPORTED), (dict(type=-1), UNSUPPORTED), (dict(param_type=1), UNSUPPORTED), (dict(act=3), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
    (dict(rows=-1), SHAPE), (dict(rows=2 ** 24 + 1), SHAPE), (dict(width=60), SHAPE), (dict(width=0), SHAPE), (dict(out_width=4), SHAPE),
    (dict(out_width=2 ** 17 + 8), SHAPE), (dict(x_stride=56), SHAPE), (dict(y_stride=120), SHAPE), (dict(x_stride=68), SHAPE), (dict(y_stride=132), SHAPE),
    (dict(x_stride=2 ** 40), SHAPE), (dict(rows_per_group=-1), SHAPE), (dict(gate_stride=120), SHAPE), (dict(gate_stride=132), SHAPE), (dict(gate_stride=2 ** 40), SHAPE)])
def test_linear_shapes(lib, kw, status):
    s = linear(**kw)
    n = C.c_size_t()
    if "gate_stride" not in kw:
        assert lib.hf_linear_workspace(C.byref(s), 0, C.byref(n)) == status and lib.hf_last_error()
    assert lib.hf_linear(C.byref(s), *[P] * 8, None) == status
    assert lib.hf_linear_backward(C.byref(s), *[P] * 10, None) == status


def test_linear_pointers(lib):
    s = linear()
    assert lib.hf_linear(None, *[P] * 8, None) == INVALID and lib.hf_linear_backward(None, *[P] * 10, None) == INVALID
    for at in range(7):         # x, weight, bias, gate, residual, y, pre
        for bad in (None, P + 8):
            if bad is None and at in (2, 3, 4, 6):
                continue
            args = [P] * 8
            args[at] = bad
            assert lib.hf_linear(C.byref(s), *args, None) == INVALID, at
    for kw in (dict(residual_stride=120), dict(residual_stride=132)):
        assert lib.hf_linear(C.byref(linear(**kw)), *[P] * 8, None) == SHAPE
    for at in range(10):        # dy, x, weight, pre, gate, dx, dweight, dbias, dgate, workspace
        for bad in (None, P + 8 if at not in (7, 8) else P + 2):
            if bad is None and at in (5, 6, 7, 8):
                continue
            args = [P] * 10
            args[at] = bad
            assert lib.hf_linear_backward(C.byref(s), *args, None) == INVALID, at       # (without a gate: dgate of nothing)
    assert lib.hf_linear_backward(C.byref(s), *[P] * 5, None, None, None, None, P, None) == 0           # nothing asked for
    assert lib.hf_linear(C.byref(linear(rows=0)), *[None] * 8, None) == 0
    n = C.c_size_t(5)
    assert lib.hf_linear_workspace(C.byref(linear(rows=0)), 1, C.byref(n)) == 0 and n.value == 0
    assert lib.hf_linear_workspace(C.byref(s), 0, None) == INVALID


def heads(pairs=(12, 10, 10), extent=(4, 4, 4), **kw):
    s = hf.hf_heads_shape(**dict(dict(type=0, param_type=0, batch=1, tokens=4, head_dim=64, heads=4, kv_heads=2, axes=3, pairing=0, over=0, eps=1e-6, pos_batch=0,
                                      rows_batch=2048, rows_token=512, grad_batch=2048, grad_token=512), **kw))
    for i, v in enumerate(pairs):
        s.pairs[i] = v
    for i, v in enumerate(extent):
        s.extent[i] = v
    t = (hf.hf_heads_tensor * 3)()
    for a in t:
        a.p, a.batch, a.token, a.head = P, 1024, 64, 256
    return s, t


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), UNSUPPORTED), (dict(param_type=1), UNSUPPORTED), (dict(pairing=2), UNSUPPORTED), (dict(over=2), UNSUPPORTED), (dict(batch=-1), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(batch=2 ** 16, tokens=2 ** 15), SHAPE), (dict(head_dim=63), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=258), SHAPE),
    (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=5), SHAPE), (dict(heads=257), SHAPE), (dict(heads=2 ** 30), SHAPE), (dict(eps=-1.0), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(axes=0), SHAPE), (dict(axes=5), SHAPE), (dict(pairs=(12, 10, 11)), SHAPE), (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2)), SHAPE),
    (dict(pairs=(-1, 1, 1)), SHAPE), (dict(extent=(4, 0, 4)), SHAPE), (dict(extent=(2 ** 31 - 1, 4, 4)), SHAPE)])
def test_heads_shapes(lib, kw, status):
    s, t = heads(**kw)
    assert lib.hf_split_heads_norm_rope(C.byref(s), *[P] * 6, t, None) == status and lib.hf_last_error()
    assert lib.hf_split_heads_norm_rope_backward(C.byref(s), t, *[P] * 10, None) == status


def test_heads_pointers(lib):
    s, t = heads()
    assert lib.hf_split_heads_norm_rope(None, *[P] * 6, t, None) == INVALID and lib.hf_split_heads_norm_rope(C.byref(s), *[P] * 6, None, None) == INVALID
    for at in range(6):         # rows, q_weight, k_weight, cos, sin, pos
        for bad in (None, P + 1):
            if bad is None and at in (1, 2):
                continue
            args = [P] * 6
            args[at] = bad
            assert lib.hf_split_heads_norm_rope(C.byref(s), *args, t, None) == INVALID, at
            assert lib.hf_split_heads_norm_rope_backward(C.byref(s), t, *args, P, P, P, P, None) == INVALID, at
    for bad in (None, P + 1):
        t[1].p = bad
        assert lib.hf_split_heads_norm_rope(C.byref(s), *[P] * 6, t, None) == INVALID
    t[1].p = P
    for at, bad in ((0, None), (0, P + 1), (1, P + 2), (2, P + 2), (3, None), (3, P + 8)):          # drows, dq_weight, dk_weight, workspace
        args = [P] * 4
        args[at] = bad
        assert lib.hf_split_heads_norm_rope_backward(C.byref(s), t, *[P] * 6, *args, None) == INVALID, at
    for kw in (dict(tokens=0), dict(batch=0)):
        s, t = heads(**kw)
        assert lib.hf_split_heads_norm_rope(C.byref(s), *[None] * 6, t, None) == 0
    assert lib.hf_split_heads_norm_rope_workspace(C.byref(heads()[0]), None) == INVALID


def test_python_refusals_without_a_device():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        layers.linear(x, torch.zeros(128, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        layers.split_heads_norm_rope(x[None], 4, 2, None, None, None, None)


def test_the_block_refuses_other_norms():
    w = gen.Workload("refusals", batch=2, heads=2, head_dim=64, tokens_per_frame=32, chunk_frames=2, window_frames=4, block=16, topk=2, keep_permille=0)
    context = types.SimpleNamespace(cfg=hf.make_config(w, merge=hf.HF_MERGE_IDENTITY), device=0)
    with pytest.raises(ValueError, match="norm_over"):
        bl.BiasedBlock(w, 4, 8, context, device="cpu", norm_over="rows")
    for over, n in (("width", 128), ("head", 64)):
        b = bl.BiasedBlock(w, 4, 8, context, device="cpu", norm_over=over)
        assert b.q_norm.shape == (n,) and b.w_first.shape == (512, 128) and not hasattr(b, "w_gate")
        with pytest.raises(ValueError, match="is taken"):
            b(torch.zeros(2, 32, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 6, 128, dtype=torch.bfloat16), b.positions(0))
