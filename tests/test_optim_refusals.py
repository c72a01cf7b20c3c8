"""What the optimizer's calls refuse, before any device call: these run without a device."""
import ctypes as C
import re

import pytest
import torch

from paper_2604_10103_b200 import binding as hf, build as hfbuild, optim
from tests.test_abi import ROOT

INVALID, SHAPE, UNSUPPORTED = 1, 2, 4
P = 0x10000            # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    hfbuild.build()
    return hf.lib()


@pytest.mark.parametrize("name", ["hf_gradient", "hf_adamw_step", "hf_adamw_tensor"])
def test_structs_match_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(f"{ROOT}/include/hf.h").read(), flags=re.S)
    body = re.findall(r"typedef struct \{([^}]*)\} " + name + ";", text)[0]
    kinds = {"int": C.c_int, "int64_t": C.c_int64, "uint32_t": C.c_uint32, "double": C.c_double}
    want = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        ty, names = re.match(r"((?:const )?\w+\*?)\s+(.*)", decl, re.S).groups()
        want += [(n.strip(), C.c_void_p if "*" in ty else kinds[ty]) for n in names.split(",")]
    assert want == list(getattr(hf, name)._fields_)


def step(**kw):
    return hf.hf_adamw_step(**dict(dict(param_type=0, grad_type=0, state_bits=32, seed=1, beta1=0.9, beta2=0.99, eps=1e-8, factor=P, counter=P), **kw))


def tensors(count=2, **kw):
    t = (hf.hf_adamw_tensor * count)()
    for a in t:
        a.p = a.g = a.master = a.m = a.v = a.scales = a.step = a.lr_at = P
        a.n = 100
    for k, v in kw.items():
        setattr(t[count - 1], k, v)
    return t


@pytest.mark.parametrize("kw,status", [
    (dict(param_type=1), UNSUPPORTED), (dict(param_type=2, grad_type=0), UNSUPPORTED), (dict(grad_type=1), UNSUPPORTED), (dict(state_bits=16), UNSUPPORTED),
    (dict(beta1=1.0), SHAPE), (dict(beta2=-0.1), SHAPE), (dict(beta1=float("nan")), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("inf")), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(factor=P + 2), INVALID), (dict(counter=None), INVALID), (dict(counter=P + 1), INVALID)])
def test_adamw_settings(lib, kw, status):
    assert lib.hf_adamw(C.byref(step(**kw)), tensors(), 2, None) == status and lib.hf_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), SHAPE), (dict(n=2 ** 44), SHAPE), (dict(p=None), INVALID), (dict(g=None), INVALID), (dict(m=None), INVALID), (dict(v=None), INVALID),
    (dict(step=None), INVALID), (dict(master=None), INVALID), (dict(p=P + 1), INVALID), (dict(g=P + 1), INVALID), (dict(master=P + 2), INVALID), (dict(m=P + 2), INVALID),
    (dict(v=P + 1), INVALID), (dict(step=P + 2), INVALID), (dict(lr_at=P + 1), INVALID)])
def test_adamw_tensors(lib, kw, status):
    assert lib.hf_adamw(C.byref(step()), tensors(**kw), 2, None) == status and lib.hf_last_error()


def test_adamw_of_eight_bits_float32_and_of_nothing(lib):
    eight = step(state_bits=8)
    for bad in (None, P + 4):
        assert lib.hf_adamw(C.byref(eight), tensors(scales=bad), 2, None) == INVALID
    assert lib.hf_adamw(C.byref(step(param_type=2, grad_type=2)), tensors(), 2, None) == INVALID           # a master of a float32 parameter
    assert lib.hf_adamw(None, tensors(), 2, None) == INVALID and lib.hf_adamw(C.byref(step()), None, 2, None) == INVALID
    assert lib.hf_adamw(C.byref(step()), tensors(), -1, None) == SHAPE
    assert lib.hf_adamw(C.byref(step()), None, 0, None) == 0
    assert lib.hf_adamw(C.byref(step(counter=None)), tensors(1, n=0, p=None, g=None, step=None), 1, None) == 0


def test_gradient_norm(lib):
    t = (hf.hf_gradient * 2)()
    for a in t:
        a.p, a.n, a.type = P, 100, 0
    call = lambda tt=t, n=2, most=1.0, out=P, ws=P: lib.hf_gradient_norm(tt, n, most, out, ws, None)  # noqa: E731
    assert call(n=-1) == SHAPE and call(tt=None) == INVALID
    assert call(most=-1.0) == SHAPE and call(most=float("nan")) == SHAPE
    assert call(out=None) == INVALID and call(out=P + 2) == INVALID and call(ws=None) == INVALID and call(ws=P + 8) == INVALID
    for k, v, status in (("type", 3, UNSUPPORTED), ("n", -1, SHAPE), ("n", 2 ** 45, SHAPE), ("p", None, INVALID), ("p", P + 1, INVALID)):
        old = getattr(t[1], k)
        setattr(t[1], k, v)
        assert call() == status, k
        setattr(t[1], k, old)
    n = C.c_size_t()
    assert lib.hf_gradient_norm_workspace(-1, C.byref(n)) == SHAPE and lib.hf_gradient_norm_workspace(1, None) == INVALID


def test_python_refusals_without_a_device():
    p = torch.nn.Parameter(torch.zeros(4))
    with pytest.raises(ValueError):
        optim.AdamW([p], state_bits=16)
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        optim.AdamW([p])
    with pytest.raises(ValueError):
        optim.gradient_norm([])
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        optim.gradient_norm([torch.zeros(3)])


def test_what_the_look_over_finds():
    """Without a device: which tensor is refused, and that nothing of it is needed for that."""
    host = hf.host()
    rows = (hf.hf_gradient * 3)()
    assert host.hf_host_gradients([], 0, rows) == 0
    assert host.hf_host_gradients([torch.zeros(3)], 0, rows) == 1                       # not on the device
    assert host.hf_host_gradients([1.0], 0, rows) == 1                                  # no tensor
    assert host.hf_host_gradients([torch.zeros(3).to_sparse()], 0, rows) == 1
    table = (hf.hf_adamw_tensor * 2)()
    sizes = (C.c_int64 * 2)(3, 3)
    p = torch.nn.Parameter(torch.zeros(3))
    assert host.hf_host_parameters([p], 0, 2, 2, sizes, table) == -1                    # no gradient
    p.grad = torch.zeros(3)
    assert host.hf_host_parameters([p], 0, 2, 2, sizes, table) == 1
    assert host.hf_host_parameters([p, p], 0, 0, 2, sizes, table) == 1
    assert host.hf_host_parameters([None], 0, 2, 2, sizes, table) == 1
    assert not table[0].p and not table[0].g
