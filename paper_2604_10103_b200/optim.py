"""The end of a training step on torch CUDA tensors: the norm of all gradients, and AdamW over many tensors at once, in one launch each (two for the
norm).  As in `layers`: calls of the library (include/hf.h) on the current device and stream, no fallback, what the library does not take raises.

    optimizer = optim.AdamW(block.parameters(), lr=1e-4, state_bits=8)
    loss.backward()
    norm, factor = optim.gradient_norm([p.grad for p in block.parameters()], max_norm=1.0)
    optimizer.step(grad_factor=factor)          # (a norm that is not finite leaves the step out; nothing waits for the device)
"""
from __future__ import annotations

import copy
import functools
import operator
import struct
from itertools import chain

import numpy as np
import torch

from . import binding as hf
from .layers import _TYPES, _check, _current, _fail, _here, _lib, _stream

_F32, _BF16 = torch.float32, torch.bfloat16
_BLOCK = 256                                                # elements that share a scale; tensors start at multiples of it in the state's buffers
_STEP = struct.Struct("@3iI3d2P").pack                      # hf_adamw_step
_rate, _of_group = operator.itemgetter("lr"), operator.itemgetter("lr", "weight_decay", "betas", "eps")
_betas = operator.itemgetter(2)                             # of those


@functools.lru_cache(maxsize=256)
def _norm_workspace(dev, n):
    return hf.hf_gradient_norm_workspace(n) // 8


def gradient_norm(tensors, max_norm=float("inf")):
    """(norm, factor), two float32 scalars on the device: the 2-norm of all tensors together (bf16, f16 or f32, contiguous, on the current device; a gradient
    that is missing, None, is left out), and min(1, max_norm / norm), which `AdamW.step` takes as its factor; NaN where the norm is not finite."""
    tensors = list(tensors)
    first = next((i for i, t in enumerate(tensors) if t is not None), None)
    if first is None:
        _fail("no tensors")
    dev = _current(f"tensors[{first}]", tensors[first])
    n = len(tensors)
    rows = bytearray(24 * n)                                # hf_gradient
    at = (hf.C.c_char * len(rows)).from_buffer(rows)
    bad = hf.host().hf_host_gradients(tensors, dev, at)
    if bad:
        t = tensors[bad - 1]
        _here(f"tensors[{bad - 1}]", t, dev)
        _fail(f"tensors[{bad - 1}] is {t.dtype}{'' if t.is_contiguous() else ', not contiguous'}: contiguous bfloat16, float16 and float32 are taken")
    out = torch.empty(2, dtype=_F32, device=tensors[first].device)
    ws = torch.empty(_norm_workspace(dev, n), dtype=torch.float64, device=out.device)
    status = _lib().hf_gradient_norm(at, n, max_norm, out.data_ptr(), ws.data_ptr(), _stream())
    if status:
        _check(status)
    return out.unbind()


def _kept(settings):
    """The settings as a copy that changes in place do not reach; None where one of them is an array or a tensor (the tables are then made anew in each step)."""
    kinds = set(map(type, chain.from_iterable(settings))) | set(map(type, chain.from_iterable(map(_betas, settings))))
    if not all(issubclass(kind, (int, float, tuple, list, np.number)) for kind in kinds):
        return None
    return settings if list not in kinds else [(lr, decay, tuple(betas) if isinstance(betas, tuple) else list(betas), eps) for lr, decay, betas, eps in settings]


class _Launch:
    """One call of the library: its parameters, and its table."""

    def __init__(self, params, sizes, dtype, grad_dtype, device, table, head, counter):
        self.params, self.dtype, self.grad_dtype, self.device, self.table, self.head, self.counter = params, dtype, grad_dtype, device, table, head, counter
        self.sizes = np.array(sizes, np.int64)
        self.at, self.look_over = table.ctypes.data, (device, _TYPES[dtype], _TYPES[grad_dtype], self.sizes.ctypes.data, table.ctypes.data)

    def look(self):
        """The parameters and gradients as they are now, into the table; otherwise (not 0) where they are not what they were."""
        return hf.host().hf_host_parameters(self.params, *self.look_over)

    def check(self):
        """The same; raises where they are not what is taken."""
        bad = self.look()
        if bad > 0:
            p = self.params[bad - 1]
            _fail(f"a parameter or its gradient is not what it was: {self.dtype} of {self.sizes[bad - 1]} elements, contiguous, on device {self.device}, and such a gradient, "
                  f"are taken, not {p.dtype} {tuple(p.shape)} on {p.device} with {p.grad.dtype} {tuple(p.grad.shape)} on {p.grad.device}")


class AdamW(torch.optim.Optimizer):
    """AdamW over bf16 and float32 parameters (contiguous, on the current device), all tensors in one launch.

    state_bits 32: moments in float32.  8: the first in e4m3, the second in e5m2, with a float32 scale for each block of 256 elements, rounded up
    or down at random by a hash of `seed`, step and place: a repeated run gives the same bits.  master_weights: a bf16 parameter has a float32
    master, from which the step starts (without one, changes below half a step of bf16 are lost); a parameter that is written from outside takes
    effect with `masters_from_parameters`.  lr may be a float32 tensor of one element on the device, which a captured step reads anew.  The tables of a step
    are kept for the next where settings and types stand still and no gradient is missing; a number in lr that changes, or a missing gradient, has them made
    anew (host time with 22 tensors 79 us instead of 15, with 132 281 instead of 24: a schedule does better to fill a tensor).

    The state lies in `buffers` (m, v, scales, master, steps), each kind in one tensor, a parameter's part at the next multiple of 256 elements;
    `state[p]` has a parameter's views.  All groups are given at construction.  A parameter without a gradient is left out of the step, and of its
    count of steps."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=32, master_weights=True, seed=0):
        if state_bits not in (8, 32):
            _fail(f"state_bits {state_bits!r}: 8 and 32 are taken")
        self._made = False
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))
        self.state_bits, self.seed = state_bits, int(seed) & 0xffffffff
        self._params = [p for g in self.param_groups for p in g["params"]]
        if len(set(self._params)) != len(self._params):         # (two parts of a launch would step it at the same time)
            _fail("a parameter is given twice")
        dev, starts, at, master_at = None, [], 0, []
        masters = 0
        for i, p in enumerate(self._params):
            dev = _current(f"parameter {i}", p)
            if p.dtype is not _F32 and p.dtype is not _BF16:
                _fail(f"parameter {i} is {p.dtype}: bfloat16 and float32 are taken")
            if not p.is_contiguous():
                _fail(f"parameter {i} has to be contiguous")
            size = -(-p.numel() // _BLOCK) * _BLOCK
            starts.append(at)
            at += size
            master_at.append(masters if master_weights and p.dtype is _BF16 else None)
            if master_at[-1] is not None:
                masters += size

        def zeros(shape, dtype):
            return torch.zeros(shape, dtype=dtype, device=self._params[0].device)
        small = state_bits == 8
        self.buffers = dict(m=zeros(at, torch.float8_e4m3fn if small else _F32), v=zeros(at, torch.float8_e5m2 if small else _F32),
                            scales=zeros((at // _BLOCK, 2), _F32) if small else None, master=zeros(masters, _F32) if masters else None,
                            steps=zeros(len(self._params) + 1, torch.int32))             # (the last: the library's counter)
        for i, (p, a, ma) in enumerate(zip(self._params, starts, master_at)):
            n = p.numel()
            s = self.state[p] = dict(step=self.buffers["steps"][i], m=self.buffers["m"][a:a + n].view(p.shape), v=self.buffers["v"][a:a + n].view(p.shape))
            if small:
                s["scales"] = self.buffers["scales"][a // _BLOCK:-(-(a + n) // _BLOCK)]
            if ma is not None:
                s["master"] = self.buffers["master"][ma:ma + n].view(p.shape)
        self._device, self._first_block = dev, [a // _BLOCK for a in starts]
        self._index, self._plan, self._planned = {p: i for i, p in enumerate(self._params)}, None, None
        # the library's table (hf_adamw_tensor) without what changes from step to step
        first, buffers = np.array(starts, np.int64), {k: b.data_ptr() for k, b in self.buffers.items() if b is not None}
        self._table = np.zeros((len(starts), 12), np.int64)
        if masters:
            self._table[:, 2] = [0 if ma is None else buffers["master"] + 4 * ma for ma in master_at]
        self._table[:, 3], self._table[:, 4] = (buffers[k] + first * (1 if small else 4) for k in ("m", "v"))
        if small:
            self._table[:, 5] = buffers["scales"] + first // _BLOCK * 8
        self._table[:, 6] = buffers["steps"] + 4 * np.arange(len(starts))
        self._table[:, 8], self._table[:, 9] = [p.numel() for p in self._params], first // _BLOCK
        self.masters_from_parameters()
        self._made = True

    def add_param_group(self, group):
        if self._made:
            _fail("all groups are given at construction: the state lies in one piece")
        super().add_param_group(group)

    def __getstate__(self):
        raise TypeError("the state lies in buffers that calls refer to: it is copied and stored by state_dict and load_state_dict")

    @torch.no_grad()
    def masters_from_parameters(self):
        """The masters of the parameters as they are now (after weights were loaded)."""
        pairs = [(self.state[p]["master"], p) for p in self._params if "master" in self.state[p]]
        if pairs:
            torch._foreach_copy_(*map(list, zip(*pairs)))

    def _rows(self, params):
        """The library's table of these parameters, without their gradients: int64 [n, 12], doubles in the last two columns."""
        table = self._table[[self._index[p] for p in params]]
        rates = {}
        for g in self.param_groups:
            lr = g["lr"]
            at = (lr.data_ptr(), 0.0) if isinstance(lr, torch.Tensor) else (0, float(lr))
            for p in g["params"]:
                rates[p] = (*at, float(g["weight_decay"]))
        table[:, 7] = [rates[p][0] for p in params]
        table[:, 10:].view(np.float64)[:] = [rates[p][1:] for p in params]
        return table

    def _launches(self, params):
        """The calls that a step over these parameters takes: those of one type, with or without masters, with the same betas and eps, together."""
        of = {p: (tuple(map(float, g["betas"])), float(g["eps"])) for g in self.param_groups for p in g["params"]}
        kinds = {}
        for p in params:
            if p.dtype is not _F32 and p.dtype is not _BF16 or p.grad.dtype is not p.dtype and p.grad.dtype is not _F32:
                _fail(f"a parameter is {p.dtype} with a gradient of {p.grad.dtype}: bfloat16 and float32 are taken, with a gradient of the same type or float32")
            kinds.setdefault((p.dtype, p.grad.dtype, "master" in self.state[p], *of[p]), []).append(p)
        for *_, (beta1, beta2), eps in kinds:       # (here, where none of the launches has run)
            if not (0.0 <= beta1 < 1.0 and 0.0 <= beta2 < 1.0 and 0.0 <= eps <= 3e38):
                _fail(f"betas {beta1}, {beta2} and eps {eps}: betas in [0, 1) and an eps >= 0, finite, are taken")
        counter = self.buffers["steps"].data_ptr() + 4 * len(self._params)
        return [_Launch(some, self._table[[self._index[p] for p in some], 8], dtype, grad_dtype, self._device, self._rows(some), (_TYPES[dtype],
                        _TYPES[grad_dtype], self.state_bits, self.seed, *betas, eps), counter) for (dtype, grad_dtype, _, betas, eps), some in kinds.items()]

    def _settings(self):
        """What the tables were made from, and step for step may change."""
        groups = self.param_groups
        if not any(issubclass(kind, torch.Tensor) for kind in set(map(type, map(_rate, groups)))):
            return list(map(_of_group, groups))
        seen = []
        for g in groups:
            lr = g["lr"]
            if isinstance(lr, torch.Tensor):
                if lr.dtype is not _F32 or lr.numel() != 1:
                    _fail("lr is a number, or a float32 tensor of one element")
                if lr.get_device() != self._device:
                    _here("lr", lr, self._device)
                lr = ("at", lr.data_ptr())
            seen.append((lr, g["weight_decay"], g["betas"], g["eps"]))
        return seen

    def step(self, closure=None, grad_factor=None):
        """One step.  grad_factor: a float32 tensor of one element on the device (as `gradient_norm` returns it), by which the gradients are
        multiplied; where it is not finite nothing is changed."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        factor = 0
        if grad_factor is not None:
            if grad_factor.dtype is not _F32 or grad_factor.numel() != 1:
                _fail("grad_factor is a float32 tensor of one element")
            if grad_factor.get_device() != self._device:
                _here("grad_factor", grad_factor, self._device)
            factor = grad_factor.data_ptr()
        _current("the first parameter", self._params[0])
        settings = self._settings()
        launches = self._plan if settings == self._planned else None
        if launches is not None and any(launch.look() for launch in launches):
            launches = None                 # (a gradient is missing, or of the other type)
        if launches is None:
            some = [p for p in self._params if p.grad is not None]
            launches = self._launches(some)
            for launch in launches:
                launch.check()
            if len(some) == len(self._params):
                self._plan, self._planned = launches, _kept(settings)
        stream = _stream()
        for launch in launches:
            status = _lib().hf_adamw(_STEP(*launch.head, factor, launch.counter), launch.at, len(launch.params), stream)
            if status:
                _check(status)
        return loss

    def state_dict(self):
        """As torch's optimizers give it, with the seed: a resumed run in 8 bits rounds as one that goes on."""
        return {**super().state_dict(), "seed": self.seed}

    @torch.no_grad()
    def load_state_dict(self, state_dict):
        """Into the state as it lies: the same parameters, state_bits and masters are taken, and refused before anything is changed otherwise.  A rate that
        lies on the device takes the saved value where it is.  The seed is the saved one, where there is one (a captured step keeps its own)."""
        state_dict = state_dict.copy()
        for hook in list(self._optimizer_load_state_dict_pre_hooks.values()):           # (torch's own method, which would call them, makes new tensors of the state)
            changed = hook(self, state_dict)
            state_dict = state_dict if changed is None else changed
        saved = state_dict["param_groups"]
        if [len(g["params"]) for g in saved] != [len(g["params"]) for g in self.param_groups]:
            _fail("the groups' numbers of parameters differ")
        ids = [i for g in saved for i in g["params"]]
        for i, p in zip(ids, self._params):
            mine, theirs = self.state[p], state_dict["state"].get(i, {})
            if mine.keys() != theirs.keys() or any(mine[k].shape != theirs[k].shape or mine[k].dtype != theirs[k].dtype for k in mine):
                _fail(f"the state of parameter {i} is of another shape, type or kind")
        for theirs in saved:
            if isinstance(theirs["lr"], torch.Tensor) and theirs["lr"].numel() != 1:
                _fail("lr is a number, or a tensor of one element")
        for i, p in zip(ids, self._params):
            for k, t in self.state[p].items():
                t.copy_(state_dict["state"][i][k])
        for mine, theirs in zip(self.param_groups, saved):
            lr, new = mine["lr"], {k: copy.deepcopy(v) for k, v in theirs.items() if k != "params"}
            if isinstance(lr, torch.Tensor):        # (where it lies: captured steps read it there)
                lr.copy_(torch.as_tensor(new["lr"]).reshape(lr.shape))
                new["lr"] = lr
            elif isinstance(new["lr"], torch.Tensor):
                new["lr"] = new["lr"].to(self.buffers["steps"].device, _F32)
            mine.update(new)
        self.seed = int(state_dict.get("seed", self.seed)) & 0xffffffff
        self._plan = self._planned = None
        for hook in list(self._optimizer_load_state_dict_post_hooks.values()):
            hook(self)
