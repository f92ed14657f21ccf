"""ctypes binding of the operators over many tensors at once (include/nuts.h, last section): argument marshalling only.

`nuts_norm` is the norm of all numbers of some tensors and the factor that bounds it; `nuts_adamw` is a step of AdamW for all parameters of a
model, whose moments a `Moments` keeps in 32 or in 8 bits.  Tensors are on the current device and without gaps.  Calls go to the streams that
those of categorical.py go to, and autograd knows none of them, either: parameters change under it as they do under `.data`.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from bisect import bisect_left
from collections import namedtuple

import torch

from . import binding as _b
from . import build as _build
from .categorical import _DTYPES, _enqueue

__all__ = ("nuts_norm", "nuts_adamw", "nuts_adamw_values", "Moments", "Norm")

Norm = namedtuple("Norm", "norm factor")

_PARAM_DTYPES = {torch.float32: _b.NUTS_F32, torch.bfloat16: _b.NUTS_BF16}
_COPY_DTYPES = {torch.bfloat16: _b.NUTS_BF16, torch.float16: _b.NUTS_F16}
TENSORS_PATH = _build.TENSORS_LIB
_PARAM, _GRAD, _COPY, _M, _V, _M_SCALE, _V_SCALE, _N = range(8)  # columns of a table of nuts_adamw_tensor
assert C.sizeof(_b.nuts_adamw_tensor) == 64 and C.sizeof(_b.nuts_tensor) == 24


_tensors = _compare = None
_SEVERAL_TYPES, _SEVERAL_DEVICES, _GAPS, _OTHER_SHAPES, _MOVED, _MEETS, _OVERLAP = 1, 2, 4, 8, 16, 32, 64


def _read(tensors, like, table, width, address, count=-1, type_=-1, kept=0):
    """Columns of `table`, rows of `width` numbers, from a list of tensors (or None); bits of what they have not in common, and of whether one lies
    in memory of `kept`."""
    global _tensors, _compare
    if _tensors is None:
        if not os.path.exists(TENSORS_PATH):
            raise ImportError(f"{TENSORS_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        if not _build.reader_fits():
            raise ImportError(f"{TENSORS_PATH} was built for another PyTorch or Python: run `python -c 'import __graft_entry__ as g; g.build()'`")
        lib = C.PyDLL(TENSORS_PATH)
        lib.nuts_tensor_table.argtypes = [C.py_object, C.py_object, C.c_void_p] + [C.c_int64] * 4 + [C.c_void_p]
        lib.nuts_tensors_compare.argtypes = [C.py_object, C.py_object]
        lib.nuts_tensor_table.restype = lib.nuts_tensors_compare.restype = C.c_int
        _tensors, _compare = lib.nuts_tensor_table, lib.nuts_tensors_compare
    return _tensors(tensors, like, table.buffer_info()[0], width, address, count, type_, kept)


def _spans(tensors):
    """Where tensors lie, in order."""
    return sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors if t is not None and t.numel())


def _meet(spans, others):
    """Whether one of `spans` has memory of one of `others`, which lie apart and in order."""
    begins = [begin for begin, _ in others]
    last = [bisect_left(begins, end) - 1 for _, end in spans]  # of the others that begin before its end
    return any(k >= 0 and others[k][1] > begin for k, (begin, _) in zip(last, spans))


def _current(device):
    """`device`, which must be the current one where there is one."""
    if torch.cuda.is_available():
        if device.type != "cuda":
            raise ValueError(f"tensors must be on the GPU, not on {device}")
        if device.index != torch.cuda.current_device():
            raise ValueError(f"tensors are on {device}, the current device is {torch.cuda.current_device()}")
    return device


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
    be multiplied with so that it is no more than max_norm (NaN where the norm is not finite in 64 bits, in which it is summed; one that 32 bits do not hold
    is infinite, and its factor is right).  None among them counts as nothing."""
    tensors = list(tensors)
    first = next((t for t in tensors if t is not None), None)
    if first is None:
        raise ValueError("nuts_norm needs a tensor")
    table = array("q", bytes(24 * len(tensors)))
    bits = _read(tensors, None, table, 3, 0, 1, 2)
    if bits & _GAPS:
        tensors = [t.contiguous() if t is not None else None for t in tensors]
        _read(tensors, None, table, 3, 0, 1, 2)
    if bits & _SEVERAL_DEVICES:
        raise ValueError("tensors must be on one device")
    if bits & _SEVERAL_TYPES and -1 in table[2::3] or first.dtype not in _DTYPES:
        raise ValueError(f"tensors must be {' or '.join(str(d) for d in _DTYPES)}")
    device = _current(first.device)
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
    parameter becomes.  states: (m, v) or (m, v, m_scales, v_scales), lists of tensors to be used for the moments.  Parameters and
    copies may be given other places later (`.data`); moments stay in the memory that they had here.  Can be copied (deeply: together with the
    parameters) and pickled."""

    def __init__(self, params, *, bits=32, copies=None, states=None):
        if bits not in (32, 8):
            raise ValueError("bits must be 32 or 8")
        self.params, self.bits = tuple(params), bits
        if not self.params:
            raise ValueError("Moments needs a parameter")
        self.dtype = self.params[0].dtype
        if self.dtype not in _PARAM_DTYPES:
            raise ValueError(f"parameters must be {' or '.join(str(d) for d in _PARAM_DTYPES)}")
        self.copies = tuple(copies) if copies is not None else (None,) * len(self.params)
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
        self.m, self.v = map(tuple, states[:2])
        self.m_scales, self.v_scales = map(tuple, states[2:]) if bits == 8 else ((None,) * n, (None,) * n)
        given = [c for c in self.copies if c is not None]
        self._first_copy = given[0] if given else None
        self.copy_dtype = given[0].dtype if given else torch.bfloat16
        if self.copy_dtype not in _COPY_DTYPES:
            raise ValueError(f"copies must be {' or '.join(str(d) for d in _COPY_DTYPES)}")
        want = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
        for i, p in enumerate(self.params):
            for t, what, dtype, size in ((p, "a parameter", self.dtype, p.numel()), (self.m[i], "m", want[0], p.numel()), (self.v[i], "v", want[1], p.numel()),
                                         (self.m_scales[i], "m_scales", torch.float32, blocks[i]), (self.v_scales[i], "v_scales", torch.float32, blocks[i]),
                                         (self.copies[i], "a copy", self.copy_dtype, p.numel())):
                if t is None and what not in ("a copy", "m_scales", "v_scales") or t is None and bits == 8 and what != "a copy":
                    raise ValueError(f"{what} of parameter {i} is missing")
                if t is not None and (t.dtype != dtype or t.numel() != size or not t.is_contiguous()):
                    raise ValueError(f"{what} of parameter {i} must be {size} {dtype} without gaps")
        self._params, self._copies = list(self.params), list(self.copies)  # (as _read wants them)
        self._sizes = [p.numel() for p in self.params]
        self._has_copies = bool(given)
        self._copy_sizes = array("q", [c.numel() if c is not None else 0 for c in self.copies])
        self._states = [[t.detach() for t in some] for some in states]  # (their memory)
        self._table = array("q", bytes(64 * n))
        self._table[_N::8] = array("q", self._sizes)
        for column, tensors in zip((_M, _V, _M_SCALE, _V_SCALE), self._states):
            _read(tensors, None, self._table, 8, column)
        self._settle()

    def __reduce__(self):
        """Copies, and what comes back from a file, have tables of their own tensors' addresses."""
        return _moments, (self.params, self.bits, self.copies if self._has_copies else None, self._states)

    def _settle(self):
        """Parameters and copies where they are now."""
        tensors = [t.detach() for some in (self.params, self.copies, *self._states) for t in some if t is not None]
        if any(t.device != self.params[0].device for t in tensors):
            raise ValueError("parameters, moments and copies must be on one device")
        self.device = _current(self.params[0].device)
        # two of them in one place would be written by two workgroups at a time
        spans = _spans(tensors)
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("parameters, moments and copies must not overlap")
        self._tensors = tensors
        self._written = array("q", [len(spans), *(at for span in spans for at in span)])
        _read(self._params, None, self._table, 8, _PARAM)
        _read(self._copies, None, self._table, 8, _COPY)

    def _now(self):
        """The table.  A parameter or a copy may have been given another place (`.data`) since: then it must still be of its kind."""
        table = self._table[:]
        bits = _read(self._params, None, table, 8, _PARAM, _N)
        if self._has_copies:
            bits |= _read(self._copies, self._params, table, 8, _COPY)
            if bits & _OTHER_SHAPES:  # (or the same number in another shape)
                bits |= _read(self._copies, None, self._copy_sizes[:], 1, -1, 0)
        # (one type for all, but is it the one?)
        if bits & (_MOVED | _GAPS | _SEVERAL_TYPES) or self.params[0].dtype is not self.dtype or self._has_copies and self._first_copy.dtype is not self.copy_dtype:
            for tensors, dtype in ((self.params, self.dtype), (self.copies, self.copy_dtype)):
                if any(t is not None and (t.numel() != n or t.dtype != dtype or t.device != self.device or not t.is_contiguous()) for t, n in zip(tensors, self._sizes)):
                    raise ValueError("a parameter or a copy has changed its size, type or device")
            self._settle()
        return table  # (calls on two threads have gradients of their own)


def _moments(params, bits, copies, states):
    return Moments(params, bits=bits, copies=copies, states=states)


def nuts_adamw(moments, grads, *, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, scale=1.0, factor=None, seed=0):
    """One step of AdamW for the parameters of `moments`, which change where they are.  grads: a tensor for each, all of one type, none of them in memory that
    the step writes (None: that parameter is left alone).  step: the step's number, from 1 on, and lr: numbers, or tensors on the device (one int64, one
    float32), which a captured step that is replayed needs.  Gradients are multiplied with scale (-1: uphill) and with factor, a float32 scalar on
    the device, of nuts_norm; where that is NaN nothing changes.  seed: of what is rounded at random (moments of 8 bits, parameters of
    bfloat16)."""
    grads = list(grads)
    if len(grads) != len(moments.params):
        raise ValueError(f"there are {len(moments.params)} parameters and {len(grads)} gradients")
    first = grads[0] if grads[0] is not None else next((g for g in grads if g is not None), None)
    if first is None:
        return
    table, dtype, device = moments._now(), first.dtype, _current(moments.device)
    written = moments._written
    bits = _read(grads, moments._params, table, 8, _GRAD, kept=written.buffer_info()[0])
    if bits & (_SEVERAL_TYPES | _SEVERAL_DEVICES | _OTHER_SHAPES) or dtype not in _DTYPES or first.device != device:
        raise ValueError(f"gradients must be {' or '.join(str(d) for d in _DTYPES)}, all of one type, on {device}, each as its parameter")
    if bits & _GAPS:
        grads = [g.contiguous() if g is not None else None for g in grads]
        bits = _read(grads, moments._params, table, 8, _GRAD, kept=written.buffer_info()[0])
    if bits & _MEETS:  # (what belongs to parameters without a gradient is not written)
        changed = [t for i, g in enumerate(grads) if g is not None for t in (moments.params[i], moments.copies[i], *(some[i] for some in moments._states))]
        if _meet(_spans(grads), _spans(changed)):
            raise ValueError("gradients must not lie in memory that the step writes")
    scalars, step_at, lr_at, factor_at = [], None, None, None
    if isinstance(step, torch.Tensor):
        scalars.append(step)
        step_at, step = _scalar(step, "step", torch.int64, device), 1
    if isinstance(lr, torch.Tensor):
        scalars.append(lr)
        lr_at, lr = _scalar(lr, "lr", torch.float32, device), 0.0
    if factor is not None:
        scalars.append(factor)
        factor_at = _scalar(factor, "factor", torch.float32, device)
    desc = _b.nuts_adamw_desc(_PARAM_DTYPES[moments.dtype], _DTYPES[dtype], _COPY_DTYPES[moments.copy_dtype], moments.bits, float(lr), float(betas[0]),
                              float(betas[1]), float(eps), float(weight_decay), float(scale), int(step), int(seed) & 0xFFFFFFFFFFFFFFFF)
    _run(_b.lib().nuts_adamw, [C.byref(desc), table.buffer_info()[0], len(grads), step_at, lr_at, factor_at], _Chain(moments._tensors, grads, scalars), device)


class _Chain:
    """Lists, one behind the other, that are gone through only where a stream has to be told of them."""

    def __init__(self, *lists):
        self.lists = lists

    def __iter__(self):
        return (t for some in self.lists for t in some)


def nuts_adamw_values(moments, *, dtype=torch.float32, out=None):
    """The moments of 8 bits as numbers: two lists of tensors (m, v), each as its parameter.  out: such lists to write to, all of one type (None for
    a tensor that is not wanted), none in memory of another or of the moments."""
    if moments.bits != 8:
        raise ValueError("moments of 32 bits are numbers: m and v")
    given = out is not None
    m, v = (list(some) for some in out) if given else ([torch.empty(p.shape, dtype=dtype, device=p.device) for p in moments.params] for _ in range(2))
    if len(m) != len(moments.params) or len(v) != len(moments.params):
        raise ValueError(f"out must be two lists of {len(moments.params)} tensors")
    first = m[0] if m[0] is not None else next((t for t in (*m, *v) if t is not None), None)
    if first is None:
        return m, v
    table, device, dtype = moments._now(), _current(moments.device), first.dtype
    written = moments._written
    kept = written.buffer_info()[0]
    bits = _read(m, moments._params, table, 8, _PARAM, kept=kept) | _read(v, moments._params, table, 8, _COPY, kept=kept)
    if given:
        bits |= _compare(m, v)
    if bits & (_SEVERAL_TYPES | _SEVERAL_DEVICES | _OTHER_SHAPES | _GAPS) or dtype not in _DTYPES or first.device != device:
        raise ValueError(f"out must be {' or '.join(str(d) for d in _DTYPES)}, all of one type, without gaps, on {device}, each as its parameter")
    if bits & _OVERLAP or bits & _MEETS and _meet(_spans([*m, *v]), _spans([t for some in moments._states for t in some])):
        raise ValueError("out must not overlap the moments, nor one of its tensors another")
    _run(_b.lib().nuts_adamw_values, [table.buffer_info()[0], len(m), _DTYPES[dtype]], _Chain(moments._tensors, m, v), device)
    return m, v
