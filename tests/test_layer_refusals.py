"""What the calls without a context refuse, before any device call: these run without a device."""
import ctypes as C
import re

import pytest
import torch

from paper_2604_10103_b200 import binding as hf, build as hfbuild, layers
from tests.test_abi import ROOT

INVALID, SHAPE, UNSUPPORTED = 1, 2, 4
P = 0x10000            # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    hfbuild.build()
    return hf.lib()


@pytest.mark.parametrize("name", ["hf_norm_shape", "hf_rope_shape", "hf_rope_tensor", "hf_ff_shape"])
def test_structs_match_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(f"{ROOT}/include/hf.h").read(), flags=re.S)
    body = re.findall(r"typedef struct \{([^}]*)\} " + name + ";", text)[0]
    want = []
    kinds = {"int": C.c_int, "int64_t": C.c_int64, "float": C.c_float, "const void*": C.c_void_p, "void*": C.c_void_p}
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        ty, names = re.match(r"(const void\*|void\*|\w+)\s+(.*)", decl, re.S).groups()
        for n in names.split(","):
            m = re.match(r"(\w+)(?:\[(\d+)\])?$", n.strip())
            want.append((m.group(1), kinds[ty] * int(m.group(2)) if m.group(2) else kinds[ty]))
    assert want == list(getattr(hf, name)._fields_)


def norm(**kw):
    return hf.hf_norm_shape(**dict(dict(type=0, param_type=0, width=64, rows=4, x_stride=64, y_stride=64, dx_stride=64, rows_per_group=0,
                                        param_stride=64, weight_offset=0.0, eps=1e-6), **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), UNSUPPORTED), (dict(param_type=1), UNSUPPORTED), (dict(type=2, param_type=0), UNSUPPORTED), (dict(width=0), SHAPE),
    (dict(width=16385, x_stride=16385, y_stride=16385), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=2 ** 31), SHAPE), (dict(x_stride=63), SHAPE),
    (dict(y_stride=8), SHAPE), (dict(rows_per_group=-1), SHAPE), (dict(rows_per_group=2, param_stride=63), SHAPE), (dict(eps=-1.0), SHAPE),
    (dict(eps=float("nan")), SHAPE)])
def test_layer_norm_shapes(lib, kw, status):
    s = norm(**kw)
    assert lib.hf_layer_norm(C.byref(s), P, P, P, P, P, P, None) == status and lib.hf_last_error()
    assert lib.hf_layer_norm_backward(C.byref(s), P, P, P, P, P, P, P, P, P, None) == status
    n = C.c_size_t()
    assert lib.hf_layer_norm_workspace(C.byref(s), C.byref(n)) == status


def test_layer_norm_pointers(lib):
    s = norm()
    assert lib.hf_layer_norm(None, P, P, P, P, P, P, None) == INVALID
    for at in (0, 3):
        args = [P] * 6
        args[at] = None
        assert lib.hf_layer_norm(C.byref(s), *args, None) == INVALID
    for at in range(6):
        args = [P] * 6
        args[at] = P + 1
        assert lib.hf_layer_norm(C.byref(s), *args, None) == INVALID
    for at in (0, 1, 2, 3):
        args = [P] * 9
        args[at] = None
        assert lib.hf_layer_norm_backward(C.byref(s), *args, None) == INVALID
    for at in range(9):
        args = [P] * 9
        args[at] = P + 1
        assert lib.hf_layer_norm_backward(C.byref(s), *args, None) == INVALID
    b = norm(dx_stride=8)
    assert lib.hf_layer_norm_backward(C.byref(b), *[P] * 9, None) == SHAPE
    assert lib.hf_layer_norm_workspace(C.byref(s), None) == INVALID
    # nothing to do is nothing done, with any pointers
    assert lib.hf_layer_norm(C.byref(norm(rows=0)), None, None, None, None, None, None, None) == 0


def rope(n=1, tensor=None, **kw):
    s = hf.hf_rope_shape(**dict(dict(type=0, batch=1, tokens=4, head_dim=64, axes=3, pairing=0, inverse=0, pos_batch=0), **{k: v for k, v in kw.items() if k not in ("pairs", "extent")}))
    for i, v in enumerate(kw.get("pairs", (12, 10, 10))):
        s.pairs[i] = v
    for i, v in enumerate(kw.get("extent", (4, 4, 4))):
        s.extent[i] = v
    t = (hf.hf_rope_tensor * 3)()
    for a in t:
        a.x, a.y, a.heads, a.rotate = P, P, 2, 1
        a.x_batch, a.x_token, a.x_head, a.y_batch, a.y_token, a.y_head = 512, 128, 64, 512, 128, 64
        for k, v in (tensor or {}).items():
            setattr(a, k, v)
    return s, t, n


@pytest.mark.parametrize("kw,status", [
    (dict(type=5), UNSUPPORTED), (dict(pairing=2), UNSUPPORTED), (dict(n=0), SHAPE), (dict(n=4), SHAPE), (dict(batch=-1), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(head_dim=63), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=1026), SHAPE), (dict(axes=0), SHAPE),
    (dict(axes=5), SHAPE), (dict(pairs=(12, 10, 11)), SHAPE), (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2)), SHAPE), (dict(pairs=(-1, 1, 1)), SHAPE),
    (dict(extent=(4, 0, 4)), SHAPE), (dict(extent=(2 ** 31 - 1, 4, 4)), SHAPE), (dict(tensor=dict(heads=-1)), SHAPE),
    (dict(tensor=dict(x=None)), INVALID), (dict(tensor=dict(y=None)), INVALID), (dict(tensor=dict(x=P + 1)), INVALID)])
def test_rope_shapes(lib, kw, status):
    s, t, n = rope(**kw)
    assert lib.hf_rope_axes(C.byref(s), t, n, P, P, P, None) == status and lib.hf_last_error()


def test_rope_pointers(lib):
    s, t, n = rope()
    assert lib.hf_rope_axes(None, t, n, P, P, P, None) == INVALID and lib.hf_rope_axes(C.byref(s), None, n, P, P, P, None) == INVALID
    for at in range(3):
        for bad in (None, P + 2):
            args = [P] * 3
            args[at] = bad
            assert lib.hf_rope_axes(C.byref(s), t, n, *args, None) == INVALID
    for kw in (dict(tokens=0), dict(batch=0), dict(tensor=dict(heads=0))):
        s, t, n = rope(**kw)
        assert lib.hf_rope_axes(C.byref(s), t, n, P, P, P, None) == 0


def ff(**kw):
    return hf.hf_ff_shape(**dict(dict(type=0, act=0, rows=4, width=64, hidden=128, out_width=64, x_stride=64, y_stride=64), **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(type=2), UNSUPPORTED), (dict(type=-1), UNSUPPORTED), (dict(act=2), UNSUPPORTED), (dict(rows=-1), SHAPE), (dict(rows=2 ** 24 + 1), SHAPE),
    (dict(width=60), SHAPE), (dict(width=0), SHAPE), (dict(hidden=4), SHAPE), (dict(out_width=12), SHAPE), (dict(hidden=2 ** 17 + 8), SHAPE),
    (dict(x_stride=56), SHAPE), (dict(y_stride=56), SHAPE), (dict(x_stride=68), SHAPE), (dict(y_stride=66), SHAPE), (dict(x_stride=2 ** 40), SHAPE)])
def test_feed_forward_shapes(lib, kw, status):
    s = ff(**kw)
    n = C.c_size_t()
    assert lib.hf_gated_ff_workspace(C.byref(s), 0, C.byref(n)) == status and lib.hf_last_error()
    assert lib.hf_gated_ff(C.byref(s), *[P] * 8, None) == status
    assert lib.hf_gated_ff_backward(C.byref(s), *[P] * 12, None) == status


def test_feed_forward_pointers(lib):
    s = ff()
    assert lib.hf_gated_ff(None, *[P] * 8, None) == INVALID and lib.hf_gated_ff_backward(None, *[P] * 12, None) == INVALID
    for at in range(8):
        for bad in (None, P + 8):
            args = [P] * 8
            args[at] = bad
            assert lib.hf_gated_ff(C.byref(s), *args, None) == INVALID, at
    for at in range(12):
        for bad in (None, P + 8):
            if at == 7 and bad is None:
                continue            # (dx may be left out)
            args = [P] * 12
            args[at] = bad
            assert lib.hf_gated_ff_backward(C.byref(s), *args, None) == INVALID, at
    assert lib.hf_gated_ff_backward(C.byref(s), *[P] * 7, None, None, None, None, P, None) == 0         # nothing asked for
    assert lib.hf_gated_ff(C.byref(ff(rows=0)), *[None] * 8, None) == 0
    assert lib.hf_gated_ff_workspace(C.byref(s), 0, None) == INVALID


def test_tensors_on_the_cpu_are_refused():
    x, w = torch.zeros(4, 64), torch.zeros(64, 64)
    tab = (torch.zeros(4), torch.zeros(4), (4,), (1,))
    pos = torch.zeros(4, 1, dtype=torch.int32)
    for call in (lambda: layers.layer_norm(x), lambda: layers.layer_norm_backward(x, x, x[:, 0], x[:, 0]),
                 lambda: layers.rope_axes(x.view(1, 4, 1, 64), pos, tab), lambda: layers.split_heads_rope(x.view(1, 4, 64), 2, 1, pos, tab),
                 lambda: layers.gated_ff(x.bfloat16(), w.bfloat16(), w.bfloat16(), w.bfloat16())):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_tensors_of_wrong_shapes_and_types_are_refused():
    x, w = torch.zeros(4, 64, device="cuda"), torch.zeros(1, 64, device="cuda")
    m, r = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    for call in (lambda: layers.layer_norm(x, w[:, :32]), lambda: layers.layer_norm(x, w, rows_per_group=2), lambda: layers.layer_norm(x, w.half()),
                 lambda: layers.layer_norm(x, w, w.half()), lambda: layers.layer_norm(x.double()), lambda: layers.layer_norm(x[:, ::2]),
                 lambda: layers.layer_norm(x.view(2, 2, 64).transpose(0, 1)), lambda: layers.layer_norm(x, w.cpu()),
                 lambda: layers.layer_norm_backward(x[:3], x, m, r), lambda: layers.layer_norm_backward(x.half(), x, m, r),
                 lambda: layers.layer_norm_backward(x, x, m[:3], r), lambda: layers.layer_norm_backward(x, x, m.half(), r)):
        with pytest.raises((ValueError, hf.HFError)):
            call()
    t, pos = (torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda"), (4,), (2,)), torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    h = x.view(1, 4, 1, 64)
    for call in (lambda: layers.rope_axes(h, pos[:3], t), lambda: layers.rope_axes(h, pos.long(), t), lambda: layers.rope_axes(h, pos, (t[0][:7],) + t[1:]),
                 lambda: layers.rope_axes(h, pos, t, pairing="third"), lambda: layers.rope_axes(h, pos, t, out=h.half()),
                 lambda: layers.rope_axes(x, pos, t), lambda: layers.rope_axes(h[..., ::2], pos, t),
                 lambda: layers.split_heads_rope(x.view(1, 4, 64), 3, 1, pos, t), lambda: layers.split_heads_rope_backward(h, h, h.half(), pos, t)):
        with pytest.raises((ValueError, hf.HFError)):
            call()
    b = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16)
    wg, wd = torch.zeros(128, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(64, 128, device="cuda", dtype=torch.bfloat16)
    for call in (lambda: layers.gated_ff(b, wg, wg[:64], wd), lambda: layers.gated_ff(b, wg, wg, wd[:, :64]), lambda: layers.gated_ff(b, wg, wg, wd, act="relu"),
                 lambda: layers.gated_ff(b.half(), wg, wg, wd), lambda: layers.gated_ff(x, wg.float(), wg.float(), wd.float()),
                 lambda: layers.gated_ff(b[:, :60], wg[:, :60].contiguous(), wg[:, :60].contiguous(), wd), lambda: layers.gated_ff(b, wd.t(), wg, wd),
                 lambda: layers.gated_ff_backward(b[:3], b, wg, wg, wd, wg[:4, :1], wg[:4])):
        with pytest.raises((ValueError, hf.HFError)):
            call()
