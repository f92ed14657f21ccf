"""ctypes binding of the categorical operators (include/nuts.h, last sections): argument marshalling only.

Where one of the sampler's targets has two classes, these operators are the parts of models with many: rows of a table by
class and their gradient, log-probabilities of given classes with entropies and alternatives, from logits or from features and
weights, and their gradients, and logits adjusted by what was said before.  Tensors are on the current device; matrices have unit stride along their rows and any from one to
the next.  A call is enqueued on the stream of nuts_set_stream, or on PyTorch's current one if that is not set, so that calls
under torch.cuda.stream() or in a torch.cuda.graph() go where PyTorch's own would.  Autograd knows none of these calls: results never
require a gradient, also where an argument does, and gradients are what the *_grad calls are asked for.
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple
from functools import lru_cache
from math import copysign

import torch

from . import binding as _b

__all__ = ("nuts_lookup", "nuts_lookup_grad", "nuts_logprobs", "nuts_logprobs_grad", "nuts_score", "nuts_score_grad",
           "Logprobs", "Scores", "nuts_penalties", "nuts_penalties_grad")

Logprobs = namedtuple("Logprobs", "logprob lse entropy top_ids top_logprobs")
Scores = namedtuple("Scores", "logprob lse entropy logits")

_DTYPES = {torch.float32: _b.NUTS_F32, torch.bfloat16: _b.NUTS_BF16, torch.float16: _b.NUTS_F16}
_ID_TYPES = {torch.int32: _b.NUTS_I32, torch.int64: _b.NUTS_I64}


# Descriptors (and the workspaces that their calls need) depend on sizes alone.
@lru_cache(maxsize=512)
def _lookup_desc(grad, sign, *fields):  # (sign: of the scale, for its zeros are equal)
    desc = _b.nuts_lookup_desc(*fields, 0)
    return C.byref(desc), _bytes(_b.lib().nuts_lookup_grad_workspace, desc) if grad else 0


@lru_cache(maxsize=512)
def _logits_desc(forward, *fields):
    desc = _b.nuts_logits_desc(*fields, 0)
    return C.byref(desc), _bytes(_b.lib().nuts_logprobs_workspace, desc) if forward else 0


@lru_cache(maxsize=512)
def _penalties_desc(grad, signs, *fields):  # (signs: of frequency and presence, for zeros are equal)
    desc = _b.nuts_penalties_desc(*fields)
    return C.byref(desc), _bytes(_b.lib().nuts_penalties_grad_workspace, desc) if grad else 0


@lru_cache(maxsize=512)
def _score_desc(grad, *fields):
    desc = _b.nuts_score_desc(*fields)
    return C.byref(desc), _bytes(_b.lib().nuts_score_grad_workspace if grad else _b.lib().nuts_score_workspace, desc)


def _bytes(query, desc):
    n = C.c_int64()
    _b._check(query(C.byref(desc), C.byref(n)))
    return n.value


def _matrix(t, what, dtypes=_DTYPES, shape=None):
    if t.dim() != 2 or t.dtype not in dtypes or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be a matrix of {' or '.join(str(d) for d in dtypes)} with unit stride along its rows")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{what} must be {shape[0]} x {shape[1]}, not {tuple(t.shape)}")
    return t


def _stride(t):
    """From row to row: of a matrix of one row or none any would do, and PyTorch's may be too small."""
    return t.stride(0) if t.shape[0] > 1 else max(1, t.shape[1])


def _ids(t, what, n=None):
    if t.dtype not in _ID_TYPES:
        raise ValueError(f"{what} must be int32 or int64")
    if n is not None and tuple(t.shape) != (n,):
        raise ValueError(f"{what} must be a vector of {n}")
    return t if t.is_contiguous() else t.contiguous()


def _in_line(t, what, ids, dim, turn=torch.Tensor.view):
    """`t`, the rows [*ids.shape, dim] of ids (or of as many ids in one line), as a matrix."""
    if t.dim() == 0 or t.shape[-1] != dim or t.numel() != ids.numel() * dim or (ids.dim() != 1 and t.shape[:-1] != ids.shape):
        raise ValueError(f"{what} must be {[*ids.shape, dim]}, not {list(t.shape)}")
    try:
        return turn(t, (ids.numel(), dim))
    except RuntimeError:  # (a view of rows that have no one distance from each other)
        raise ValueError(f"{what} must have its rows at one distance from each other") from None


def _per_row(t, what, n):
    if t is None:
        return None
    if t.dtype != torch.float32 or tuple(t.shape) != (n,):
        raise ValueError(f"{what} must be a float32 vector of {n}")
    return t if t.is_contiguous() else t.contiguous()


def _call(entry, desc, tensors, workspace_bytes=None, last=()):
    """`entry` of a descriptor and `tensors`, its pointers in order (None: NULL), then the workspace."""
    device = tensors[0].device
    args = [desc]
    for t in tensors:
        if t is None:
            args.append(None)
        elif t.device == device:
            args.append(t.data_ptr())
        else:
            raise ValueError(f"tensors are on {device} and {t.device}")
    if device.type != "cuda":
        if torch.cuda.is_available():
            raise ValueError(f"tensors must be on the GPU, not on {device}")
        # no device: the library says so itself
        _b._check(entry(*args, *((256, 1 << 62) if workspace_bytes is not None else ()), *last))
        return
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is {torch.cuda.current_device()}")
    if workspace_bytes is not None:
        workspace = torch.empty(workspace_bytes, dtype=torch.uint8, device=device) if workspace_bytes else None
        args += (workspace.data_ptr() if workspace_bytes else None, workspace_bytes)
        tensors = (*tensors, workspace)
    _enqueue(entry, args + list(last), tensors, device)


def _enqueue(entry, args, tensors, device):
    """`entry` on the library's stream, or PyTorch's current one; `tensors`: all that it uses."""
    current = torch._C._cuda_getCurrentRawStream(device.index)
    own = getattr(_b._thread, "stream", 0)
    if own and own != current:
        # PyTorch's allocator learns that the library's stream uses these, and the stream waits for what PyTorch's has made
        stream = torch.cuda.ExternalStream(own, device=device)
        stream.wait_stream(torch.cuda.current_stream(device))
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        _b._check(entry(*args))
    elif own or not current:
        _b._check(entry(*args))
    else:
        L = _b.lib()
        L.nuts_set_stream(current)
        try:
            _b._check(entry(*args))
        finally:
            L.nuts_set_stream(None)


def nuts_lookup(table, ids, *, scale=1.0, out=None):
    """scale * table[ids]: [*ids.shape, dim], zeros where an id is no row of the table."""
    _matrix(table, "table")
    ids = _ids(ids, "ids")
    classes, dim = table.shape
    n = ids.numel()
    if out is None:
        out = table.new_empty((*ids.shape, dim))
    elif out.dtype != table.dtype:
        raise ValueError(f"out must be {table.dtype}")
    rows = _matrix(out if out.dim() == 2 else _in_line(out, "out", ids, dim), "out", shape=(n, dim))
    scale = float(scale)
    desc, _ = _lookup_desc(False, copysign(1.0, scale), _DTYPES[table.dtype], _ID_TYPES[ids.dtype], n, classes, dim, _stride(table),
                           _stride(rows), scale, 0)
    _call(_b.lib().nuts_lookup, desc, (table, ids, rows))
    return out


def nuts_lookup_grad(grad, ids, n_classes, *, scale=1.0, out=None, accumulate=False):
    """Gradient of nuts_lookup with respect to its table [n_classes, dim], from that with respect to its rows, `grad`
    [*ids.shape, dim].  accumulate: it is added to `out`, and rows of classes that do not come are not touched."""
    ids = _ids(ids, "ids")
    n, dim = ids.numel(), grad.shape[-1] if grad.dim() else 0
    rows = _matrix(grad if grad.dim() == 2 else _in_line(grad, "grad", ids, dim, torch.Tensor.reshape), "grad", shape=(n, dim))
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = grad.new_empty((n_classes, dim))
    elif out.dtype != grad.dtype:
        raise ValueError(f"out must be {grad.dtype}")
    _matrix(out, "out", shape=(n_classes, dim))
    scale = float(scale)
    desc, size = _lookup_desc(True, copysign(1.0, scale), _DTYPES[grad.dtype], _ID_TYPES[ids.dtype], n, n_classes, dim, _stride(out),
                              _stride(rows), scale, int(bool(accumulate)))
    _call(_b.lib().nuts_lookup_grad, desc, (rows, ids, out), size)
    return out


def _mask(allowed, n, classes):
    """(tensor, words from row to row) of a mask: [words] for all rows or [n, words]."""
    if allowed is None:
        return None, 0
    words = (classes + 31) // 32
    if allowed.dtype != torch.int32 or allowed.shape[-1] != words or allowed.dim() > 2 or (words > 1 and allowed.stride(-1) != 1):
        raise ValueError(f"allowed must be int32 [{words}] or [{n}, {words}]: bit v % 32 of word v / 32 is class v's")
    if allowed.dim() == 1 or (allowed.shape[0] == 1 and n != 1):
        return allowed, 0
    if allowed.shape[0] != n:
        raise ValueError(f"allowed must be int32 [{words}] or [{n}, {words}]")
    return allowed, allowed.stride(0) if n > 1 else words


def nuts_logprobs(logits, targets=None, *, scale=1.0, allowed=None, n_top=0):
    """Log-probabilities of `targets` under softmax(scale * logits), row by row, with the logarithm of the sum, the entropy and the
    n_top most probable classes.  allowed: bits, of the classes that may come ([words], or [rows, words])."""
    _matrix(logits, "logits")
    n, classes = logits.shape
    id_type = _b.NUTS_I32
    if targets is not None:
        targets = _ids(targets, "targets", n)
        id_type = _ID_TYPES[targets.dtype]
    allowed, allowed_stride = _mask(allowed, n, classes)
    desc, size = _logits_desc(True, _DTYPES[logits.dtype], id_type, n, classes, _stride(logits), allowed_stride, float(scale), int(n_top))
    logprob, lse, entropy = torch.empty((3, n), dtype=torch.float32, device=logits.device).unbind(0)
    top_ids = top_logprobs = None
    if n_top:
        top_ids = torch.empty((n, n_top), dtype=torch.int32, device=logits.device)
        top_logprobs = torch.empty((n, n_top), dtype=torch.float32, device=logits.device)
    _call(_b.lib().nuts_logprobs, desc, (logits, targets, allowed, logprob, lse, entropy, top_ids, top_logprobs), size)
    return Logprobs(logprob if targets is not None else None, lse, entropy, top_ids, top_logprobs)


def nuts_logprobs_grad(logits, targets, lse, entropy=None, *, grad_logprob=None, grad_lse=None, grad_entropy=None, scale=1.0,
                       allowed=None, out=None):
    """Gradient with respect to the logits, from the gradients with respect to nuts_logprobs' outputs."""
    _matrix(logits, "logits")
    n, classes = logits.shape
    id_type = _b.NUTS_I32
    if targets is not None:
        targets = _ids(targets, "targets", n)
        id_type = _ID_TYPES[targets.dtype]
    allowed, allowed_stride = _mask(allowed, n, classes)
    desc, _ = _logits_desc(False, _DTYPES[logits.dtype], id_type, n, classes, _stride(logits), allowed_stride, float(scale), 0)
    if out is None:
        out = logits.new_empty((n, classes))
    elif out.dtype != logits.dtype:
        raise ValueError(f"out must be {logits.dtype}")
    _matrix(out, "out", shape=(n, classes))
    _call(_b.lib().nuts_logprobs_grad, desc,
          (logits, targets, allowed, _per_row(lse, "lse", n), _per_row(entropy, "entropy", n), _per_row(grad_logprob, "grad_logprob", n),
           _per_row(grad_lse, "grad_lse", n), _per_row(grad_entropy, "grad_entropy", n), out), last=(_stride(out),))
    return out


_SCORE_DTYPES = {torch.float32: _b.NUTS_F32, torch.bfloat16: _b.NUTS_BF16}


def _score_args(x, weight, targets):
    _matrix(x, "x", _SCORE_DTYPES)
    _matrix(weight, "weight", _SCORE_DTYPES)
    if weight.dtype != x.dtype or weight.shape[1] != x.shape[1]:
        raise ValueError(f"weight must be {x.dtype} with {x.shape[1]} columns, as x")
    id_type = _b.NUTS_I32
    if targets is not None:
        targets = _ids(targets, "targets", x.shape[0])
        id_type = _ID_TYPES[targets.dtype]
    # (the library takes matrices that begin at multiples of 16 bytes)
    x, weight = (t.clone() if t.data_ptr() % 16 else t for t in (x, weight))
    return x, weight, targets, (_SCORE_DTYPES[x.dtype], id_type, x.shape[0], weight.shape[0], x.shape[1], _stride(x), _stride(weight))


def nuts_score(x, weight, targets=None, *, scale=1.0, keep_logits=False):
    """nuts_logprobs of the logits scale * x @ weight.T, which are not stored unless keep_logits: then they are returned, too, in
    binary32, for nuts_score_grad (which otherwise computes them again) or for nuts_logprobs to name alternatives."""
    x, weight, targets, fields = _score_args(x, weight, targets)
    n, classes = x.shape[0], weight.shape[0]
    # rows of whole cache lines
    logits = torch.empty((n, (classes + 31) // 32 * 32), dtype=torch.float32, device=x.device)[:, :classes] if keep_logits else None
    desc, size = _score_desc(False, *fields, _stride(logits) if keep_logits else classes, x.shape[1], x.shape[1], float(scale))
    logprob, lse, entropy = torch.empty((3, n), dtype=torch.float32, device=x.device).unbind(0)
    _call(_b.lib().nuts_score, desc, (x, weight, targets, logprob, lse, entropy, logits), size)
    return Scores(logprob if targets is not None else None, lse, entropy, logits)


def nuts_score_grad(x, weight, targets, lse, entropy=None, *, grad_logprob=None, grad_lse=None, grad_entropy=None, scale=1.0,
                    logits=None, want_x=True, want_weight=True):
    """(gradient with respect to x, gradient with respect to weight), from the gradients with respect to nuts_score's outputs;
    None for one that is not wanted."""
    x, weight, targets, fields = _score_args(x, weight, targets)
    n, classes = x.shape[0], weight.shape[0]
    if logits is not None:
        _matrix(logits, "logits", {torch.float32: 0}, (n, classes))
    grad_x = x.new_empty((n, x.shape[1])) if want_x else None
    grad_weight = x.new_empty((classes, x.shape[1])) if want_weight else None
    desc, size = _score_desc(True, *fields, _stride(logits) if logits is not None else classes, x.shape[1], x.shape[1], float(scale))
    _call(_b.lib().nuts_score_grad, desc,
          (x, weight, targets, logits, _per_row(lse, "lse", n), _per_row(entropy, "entropy", n), _per_row(grad_logprob, "grad_logprob", n),
           _per_row(grad_lse, "grad_lse", n), _per_row(grad_entropy, "grad_entropy", n), grad_x, grad_weight), size)
    return grad_x, grad_weight


def _factor(value, what, n, device):
    """(number of all rows, tensor of each row's) of a penalty's strength."""
    if type(value) is not float and isinstance(value, torch.Tensor) and value.dim() > 0:
        return 1.0, _per_row(value, what, n)
    return float(value), None


def _places(t, what, n):
    if t is None:
        return None
    if t.dtype != torch.int32 or tuple(t.shape) != (n,):
        raise ValueError(f"{what} must be an int32 vector of {n}")
    return t if t.is_contiguous() else t.contiguous()


def _history(t, n):
    """(tensor, type, places in a row, from row to row) of the classes said before: [places] for all rows or [n, places]."""
    if t is None:
        return None, None, 0, 0
    shape, id_type = t.shape, _ID_TYPES.get(t.dtype)
    if len(shape) == 2 and shape[0] in (1, n):
        rows, places = shape
        apart, step = t.stride()
    elif len(shape) == 1:
        rows, places, apart, step = 1, shape[0], 0, t.stride(0)
    else:
        id_type = None
    if id_type is None:
        raise ValueError(f"history must be int32 or int64 [places] or [{n}, places]")
    if (places > 1 and step != 1) or (rows > 1 and 0 < apart < places):  # (rows that overlap, too)
        t = t.contiguous()
        apart = places
    return t, id_type, places, apart if rows > 1 else 0


def _rows_like(logits):
    """New rows of the shape of `logits`, which begin at whole cache lines where they are long: written so they take a sixth less time than
    odd ones that follow each other."""
    n, classes = logits.shape
    line = 128 // logits.element_size()
    if n <= 1 or classes < 1024 or classes % line == 0:
        return torch.empty((n, classes), dtype=logits.dtype, device=logits.device)
    return torch.empty((n, (classes + line - 1) // line * line), dtype=logits.dtype, device=logits.device)[:, :classes]


def nuts_penalties(logits, history=None, *, lengths=None, prompts=None, repetition=1.0, frequency=0.0, presence=0.0, bias=None,
                   bias_ids=None, bias_values=None, allowed=None, out=None):
    """Logits of which classes that came in a row's history are penalised, to which biases are added, and in which classes that may not
    come are -infinity.  history: [places] for all rows or [rows, places], of which the first lengths[row] are there, and the
    first prompts[row] are not the model's own.  repetition, frequency, presence: numbers, or a float32 vector of each row's.
    bias: float32 [classes] or [rows, classes]; bias_ids, bias_values: [rows, some], biases of single classes.  allowed: bits, as in
    nuts_logprobs.  out: where to write, which may be `logits`; a new one's rows may lie further apart than they are long."""
    _matrix(logits, "logits")
    n, classes = logits.shape
    history, id_type, places, history_stride = _history(history, n)
    if out is None:
        out = _rows_like(logits)
    elif out.dtype != logits.dtype:
        raise ValueError(f"out must be {logits.dtype}")
    _matrix(out, "out", shape=(n, classes))
    n_bias = 0
    if (bias_ids is None) != (bias_values is None):
        raise ValueError("bias_ids and bias_values need each other")
    if bias_ids is not None:
        if bias_ids.dtype not in _ID_TYPES or bias_ids.dim() != 2 or bias_ids.shape[0] != n:
            raise ValueError(f"bias_ids must be int32 or int64 [{n}, some]")
        if bias_values.dtype != torch.float32 or bias_values.shape != bias_ids.shape:
            raise ValueError(f"bias_values must be float32 {list(bias_ids.shape)}")
        if id_type is None:
            id_type = _ID_TYPES[bias_ids.dtype]
        elif id_type != _ID_TYPES[bias_ids.dtype]:  # (to the wider type: the other could make a class of what is none)
            history, id_type, places, history_stride = _history(history.long(), n)  # (which may be another tensor, or the same)
            bias_ids = bias_ids.long()
        bias_ids, bias_values, n_bias = bias_ids.contiguous(), bias_values.contiguous(), bias_ids.shape[1]
    bias_stride = 0
    if bias is not None:
        if bias.dtype != torch.float32 or tuple(bias.shape) not in ((classes,), (1, classes), (n, classes)) or (classes > 1 and bias.stride(-1) != 1):
            raise ValueError(f"bias must be float32 [{classes}] or [{n}, {classes}] with unit stride along its rows")
        if bias.dim() == 2 and bias.shape[0] > 1 and bias.stride(0):
            bias_stride = bias.stride(0)
    allowed, allowed_stride = _mask(allowed, n, classes)
    r, rs = _factor(repetition, "repetition", n, logits.device)
    f, fs = _factor(frequency, "frequency", n, logits.device)
    q, qs = _factor(presence, "presence", n, logits.device)
    desc, _ = _penalties_desc(False, (copysign(1.0, f), copysign(1.0, q)), _DTYPES[logits.dtype], _b.NUTS_I32 if id_type is None else id_type, n, classes,
                              _stride(logits), _stride(out), allowed_stride, bias_stride, places, history_stride, n_bias, r, f, q)
    _call(_b.lib().nuts_penalties, desc,
          (logits, history, _places(lengths, "lengths", n), _places(prompts, "prompts", n), rs, fs, qs, bias, bias_ids, bias_values, allowed, out))
    return out


def nuts_penalties_grad(grad, logits, history=None, *, lengths=None, repetition=1.0, allowed=None, out=None, want_logits=True, want_bias=False):
    """(gradient with respect to the logits, gradient with respect to a bias [classes] that all rows share), from `grad`, that with
    respect to what nuts_penalties gave for `logits`; None for one that is not wanted.  out: where to write the first, which may be `grad`.
    (With respect to a bias of each row it is `grad` where classes are allowed.)"""
    _matrix(logits, "logits")
    n, classes = logits.shape
    if grad.dtype != logits.dtype:
        raise ValueError(f"grad must be {logits.dtype}")
    _matrix(grad, "grad", shape=(n, classes))
    history, id_type, places, history_stride = _history(history, n)
    if not want_logits:
        if out is not None:
            raise ValueError("out is for the gradient with respect to the logits")
    elif out is None:
        out = _rows_like(logits)
    elif out.dtype != logits.dtype:
        raise ValueError(f"out must be {logits.dtype}")
    if out is not None:
        _matrix(out, "out", shape=(n, classes))
    grad_bias = torch.empty(classes, dtype=torch.float32, device=logits.device) if want_bias else None
    allowed, allowed_stride = _mask(allowed, n, classes)
    r, rs = _factor(repetition, "repetition", n, logits.device)
    desc, size = _penalties_desc(want_bias, (1.0, 1.0), _DTYPES[logits.dtype], _b.NUTS_I32 if id_type is None else id_type, n, classes, _stride(logits),
                                 _stride(out) if out is not None else classes, allowed_stride, 0, places, history_stride, 0, r, 0.0, 0.0)
    lengths = _places(lengths, "lengths", n)
    L = _b.lib()
    _call(lambda desc, g, *rest: L.nuts_penalties_grad(desc, g, _stride(grad), *rest), desc,
          (grad, logits, history, lengths, rs, allowed, out, grad_bias), size)
    return out, grad_bias
