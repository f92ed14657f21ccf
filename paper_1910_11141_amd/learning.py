"""ctypes binding of the operators over many tensors at once (include/nuts.h, last section): argument marshalling only.

`nuts_norm` is the norm of all numbers of some tensors and the factor that bounds it; `nuts_adamw` is a step of AdamW for all parameters of a
model, whose moments a `Moments` keeps in 32 or in 8 bits.  Tensors are on the current device and without gaps.  Calls go to the streams that
those of categorical.py go to, and autograd knows none of them, either: parameters change under it as they do under `.data`.
"""
from __future__ import annotations

import ctypes as C
from array import array
from collections import namedtuple

import torch

from . import binding as _b
from .categorical import _DTYPES, _enqueue

__all__ = ("nuts_norm", "nuts_adamw", "nuts_adamw_values", "Moments", "Norm")

Norm = namedtuple("Norm", "norm factor")

_PARAM_DTYPES = {torch.float32: _b.NUTS_F32, torch.bfloat16: _b.NUTS_BF16}
_COPY_DTYPES = {torch.bfloat16: _b.NUTS_BF16, torch.float16: _b.NUTS_F16}
_PARAM, _GRAD, _COPY, _M, _V, _M_SCALE, _V_SCALE, _N = range(8)  # columns of a table of nuts_adamw_tensor
assert C.sizeof(_b.nuts_adamw_tensor) == 64 and C.sizeof(_b.nuts_tensor) == 24


def _of_one_device(tensors):
    """The device of `tensors` (None where there are none), which must be the current one."""
    device = tensors[0].device if tensors else None
    if device is not None and any([t.get_device() != device.index for t in tensors] if device.type == "cuda" else [t.device != device for t in tensors]):
        raise ValueError(f"tensors are on {' and '.join(sorted({str(t.device) for t in tensors}))}")
    if device is not None and torch.cuda.is_available():
        if device.type != "cuda":
            raise ValueError(f"tensors must be on the GPU, not on {device}")
        if device.index != torch.cuda.current_device():
            raise ValueError(f"tensors are on {device}, the current device is {torch.cuda.current_device()}")
    return device


def _places(tensors):
    return array("q", [t.data_ptr() if t is not None else 0 for t in tensors])


def _run(entry, args, tensors, device):
    if device is None or device.type != "cuda":
        _b._check(entry(*args))  # no device: the library says so itself
    else:
        _enqueue(entry, args, tensors, device)


def _scalar(t, what, dtype, device):
    """A scalar that stays on the device."""
    if t.dtype != dtype or t.numel() != 1:
        raise ValueError(f"{what} must be one {dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"tensors are on {device} and {t.device}")
    return t.data_ptr()


def nuts_norm(tensors, *, max_norm=1.0):
    """(norm, factor), float32 scalars on the device: the square root of the sum of all squares of `tensors`, and what all of them are to
    be multiplied with so that it is no more than max_norm (NaN where the norm is not finite)."""
    tensors = [t if t.is_contiguous() else t.contiguous() for t in tensors]
    device = _of_one_device(tensors)
    if device is None:
        raise ValueError("nuts_norm needs a tensor")
    try:
        table = array("q", [x for t in tensors for x in (t.data_ptr(), t.numel(), _DTYPES[t.dtype])])  # (0 behind the type)
    except KeyError as e:
        raise ValueError(f"tensors must be {' or '.join(str(d) for d in _DTYPES)}, not {e.args[0]}") from None
    L, size, at = _b.lib(), C.c_int64(), table.buffer_info()[0]
    _b._check(L.nuts_norm_workspace(at, len(tensors), C.byref(size)))
    norm, factor = torch.empty(2, dtype=torch.float32, device=device).unbind(0)
    workspace = torch.empty(size.value, dtype=torch.uint8, device=device) if size.value and device.type == "cuda" else None
    _run(L.nuts_norm, [at, len(tensors), float(max_norm), norm.data_ptr(), factor.data_ptr(),
                       workspace.data_ptr() if workspace is not None else 256, size.value], [*tensors, norm, workspace], device)
    return Norm(norm, factor)


class Moments:
    """What AdamW keeps of a list of parameters (all float32, or all bfloat16): their moments, zeros at first, in 32 bits
    (`m`, `v`: float32, as the parameters) or in 8 (`m` int8, `v` uint8, as the parameters; `m_scales`, `v_scales`: float32, one for each 256 of a
    parameter's numbers).  copies: a tensor of bfloat16 or float16 for each parameter (or None), which receives what the
    parameter becomes.  states: (m, v) or (m, v, m_scales, v_scales), lists of tensors to be used for the moments."""

    def __init__(self, params, *, bits=32, copies=None, states=None):
        if bits not in (32, 8):
            raise ValueError("bits must be 32 or 8")
        self.params, self.bits = list(params), bits
        if not self.params:
            raise ValueError("Moments needs a parameter")
        self.dtype = self.params[0].dtype
        if self.dtype not in _PARAM_DTYPES:
            raise ValueError(f"parameters must be {' or '.join(str(d) for d in _PARAM_DTYPES)}")
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        n = len(self.params)
        blocks = [-(-p.numel() // _b.NUTS_STATE_BLOCK) for p in self.params]
        if states is None:
            kinds = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
            states = [[torch.zeros(p.shape, dtype=k, device=p.device) for p in self.params] for k in kinds]
            if bits == 8:
                states += [[torch.zeros(b, dtype=torch.float32, device=p.device) for b, p in zip(blocks, self.params)] for _ in range(2)]
        states = [list(s) for s in states]
        if len(states) != (2 if bits == 32 else 4) or any(len(s) != n for s in states) or len(self.copies) != n:
            raise ValueError(f"states must be {'(m, v)' if bits == 32 else '(m, v, m_scales, v_scales)'}, and they and copies must have {n} tensors each")
        self.m, self.v = states[:2]
        self.m_scales, self.v_scales = states[2:] if bits == 8 else ([None] * n, [None] * n)
        given = [c for c in self.copies if c is not None]
        self.copy_dtype = given[0].dtype if given else torch.bfloat16
        if self.copy_dtype not in _COPY_DTYPES:
            raise ValueError(f"copies must be {' or '.join(str(d) for d in _COPY_DTYPES)}")
        want = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
        for i, p in enumerate(self.params):
            for t, what, dtype, size in ((p, "a parameter", self.dtype, p.numel()), (self.m[i], "m", want[0], p.numel()), (self.v[i], "v", want[1], p.numel()),
                                         (self.m_scales[i], "m_scales", torch.float32, blocks[i]), (self.v_scales[i], "v_scales", torch.float32, blocks[i]),
                                         (self.copies[i], "a copy", self.copy_dtype, p.numel())):
                if t is not None and (t.dtype != dtype or t.numel() != size or not t.is_contiguous()):
                    raise ValueError(f"{what} of parameter {i} must be {size} {dtype} without gaps")
        self._tensors = [t for each in zip(self.params, self.copies, *states) for t in each if t is not None]
        self.device = _of_one_device(self._tensors)
        self._describe()
        # two of them in one place would be written by two workgroups at a time
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self._tensors if t.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("parameters, moments and copies must not overlap")

    def _describe(self):
        self._sizes, self._shapes = [p.numel() for p in self.params], [p.shape for p in self.params]
        self._table = array("q", bytes(64 * len(self.params)))
        for column, tensors in ((_PARAM, self.params), (_COPY, self.copies), (_M, self.m), (_V, self.v), (_M_SCALE, self.m_scales), (_V_SCALE, self.v_scales)):
            self._table[column::8] = _places(tensors)
        self._table[_N::8] = array("q", self._sizes)
        self._at = self._table[_PARAM::8].tolist()

    def _check_places(self):
        """A parameter may have been given another place (`.data`) since: then it must still be of its kind."""
        if [p.data_ptr() for p in self.params] != self._at:
            if any(p.numel() != n or p.dtype != self.dtype or p.device != self.device or not p.is_contiguous() for p, n in zip(self.params, self._sizes)):
                raise ValueError("a parameter has changed its size, type or device")
            self.__init__(self.params, bits=self.bits, copies=None if all(c is None for c in self.copies) else self.copies,
                          states=(self.m, self.v) if self.bits == 32 else (self.m, self.v, self.m_scales, self.v_scales))


def nuts_adamw(moments, grads, *, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, scale=1.0, factor=None, seed=0):
    """One step of AdamW for the parameters of `moments`, which change where they are.  grads: a tensor for each, all of one type (None: that
    parameter is left alone).  step: the step's number, from 1 on, and lr: numbers, or tensors on the device (one int64, one
    float32), which a captured step that is replayed needs.  Gradients are multiplied with scale (-1: uphill) and with factor, a float32 scalar on
    the device, of nuts_norm; where that is NaN nothing changes.  seed: of what is rounded at random (moments of 8 bits, parameters of
    bfloat16)."""
    grads = list(grads)
    if len(grads) != len(moments.params):
        raise ValueError(f"there are {len(moments.params)} parameters and {len(grads)} gradients")
    moments._check_places()
    device, used = moments.device, [g for g in grads if g is not None]
    if not used:
        return
    dtype = used[0].dtype
    if dtype not in _DTYPES:
        raise ValueError(f"gradients must be {' or '.join(str(d) for d in _DTYPES)}")
    at = used[0].get_device()
    if used[0].device != device or any([g is not None and (g.shape != shape or g.dtype is not dtype or g.get_device() != at) for g, shape in zip(grads, moments._shapes)]):
        raise ValueError(f"gradients must be {dtype} on {device}, each as its parameter")
    if not all([g.is_contiguous() for g in used]):
        grads = [g.contiguous() if g is not None else None for g in grads]
        used = [g for g in grads if g is not None]
    places = _places(grads)
    if device.type == "cuda" and device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is {torch.cuda.current_device()}")
    step_at = lr_at = factor_at = None
    if isinstance(step, torch.Tensor):
        step_at, step = _scalar(step, "step", torch.int64, device), used.append(step) or 1
    if isinstance(lr, torch.Tensor):
        lr_at, lr = _scalar(lr, "lr", torch.float32, device), used.append(lr) or 0.0
    if factor is not None:
        factor_at = _scalar(factor, "factor", torch.float32, device)
        used.append(factor)
    table = moments._table[:]  # (calls on two threads have gradients of their own)
    table[_GRAD::8] = places
    desc = _b.nuts_adamw_desc(_PARAM_DTYPES[moments.dtype], _DTYPES[dtype], _COPY_DTYPES[moments.copy_dtype], moments.bits, float(lr), float(betas[0]),
                              float(betas[1]), float(eps), float(weight_decay), float(scale), int(step), int(seed) & 0xFFFFFFFFFFFFFFFF)
    _run(_b.lib().nuts_adamw, [C.byref(desc), table.buffer_info()[0], len(grads), step_at, lr_at, factor_at], _Both(moments._tensors, used), device)


class _Both:
    """Two lists, one behind the other, that are gone through only where a stream has to be told of them."""

    def __init__(self, *lists):
        self.lists = lists

    def __iter__(self):
        return (t for some in self.lists for t in some)


def nuts_adamw_values(moments, *, dtype=torch.float32, out=None):
    """The moments of 8 bits as numbers: two lists of tensors (m, v), each as its parameter.  out: such lists to write to, all of one type (None for
    a tensor that is not wanted)."""
    if moments.bits != 8:
        raise ValueError("moments of 32 bits are numbers: m and v")
    if out is None:
        out = tuple([torch.empty(p.shape, dtype=dtype, device=p.device) for p in moments.params] for _ in range(2))
    m, v = (list(some) for some in out)
    if len(m) != len(moments.params) or len(v) != len(moments.params):
        raise ValueError(f"out must be two lists of {len(moments.params)} tensors")
    used = [t for t in (*m, *v) if t is not None]
    if not used:
        return m, v
    dtype, at = used[0].dtype, used[0].get_device()
    if dtype not in _DTYPES or used[0].device != moments.device or any(
            [t is not None and (t.numel() != n or t.dtype is not dtype or t.get_device() != at or not t.is_contiguous()) for some in (m, v) for t, n in zip(some, moments._sizes)]):
        raise ValueError(f"out must be {' or '.join(str(d) for d in _DTYPES)} without gaps on {moments.device}, each as its parameter")
    if moments.device.type == "cuda" and moments.device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {moments.device}, the current device is {torch.cuda.current_device()}")
    table = moments._table[:]
    table[_PARAM::8], table[_COPY::8] = _places(m), _places(v)
    _run(_b.lib().nuts_adamw_values, [table.buffer_info()[0], len(m), _DTYPES[dtype]], _Both(moments._tensors, used), moments.device)
    return m, v
