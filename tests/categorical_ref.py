"""Plain forms of the categorical operators in 64 bits (PyTorch, any device), and bounds of what 32-bit sums may be off by."""
import math

import numpy as np
import torch

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a unit in the last of 24, 8 and 11 places
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}  # and where there are no more places
U = 2.0 ** -24


def lookup_grad(grad, ids, n_classes, scale, old=None):
    """(sums, bound): a class's rows added up in 64 bits; a 32-bit sum of c terms in any order is off by at most
    (c - 1) u sum |terms|, and two products or sums with the scale and what was there follow."""
    n, dim = grad.shape
    known = (ids >= 0) & (ids < n_classes)
    at, rows = ids[known].long(), grad[known].double()
    out = torch.zeros(n_classes, dim, dtype=torch.float64, device=grad.device).index_add_(0, at, rows)
    size = torch.zeros_like(out).index_add_(0, at, rows.abs())
    count = torch.zeros(n_classes, dtype=torch.float64, device=grad.device).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    out, bound = out * scale, (count[:, None] + 2) * U * size * abs(scale)
    if old is not None:
        out = out + old.double()
        bound = bound + U * old.double().abs()
    return out, bound + (out.abs() + bound) * EPS[grad.dtype] * 1.01 + TINY[grad.dtype]


def bits(allowed, classes):
    """[.., words] of int32 as booleans [.., classes]."""
    shifts = torch.arange(32, device=allowed.device, dtype=torch.int32)
    return ((allowed[..., None] >> shifts) & 1).flatten(-2)[..., :classes].bool()


def pack_bits(mask):
    """Booleans [.., classes] as int32 [.., words]."""
    classes = mask.shape[-1]
    words = (classes + 31) // 32
    padded = torch.zeros(*mask.shape[:-1], words * 32, dtype=torch.int64, device=mask.device)
    padded[..., :classes] = mask
    value = (padded.view(*mask.shape[:-1], words, 32) << torch.arange(32, device=mask.device)).sum(-1)
    return torch.where(value >= 2 ** 31, value - 2 ** 32, value).int()


def logprobs(z, targets):
    """(logprob, lse, entropy, p) of rows of z (64 bits, -inf where a class may not come), as the header defines them."""
    n, classes = z.shape
    m = z.amax(1, keepdim=True)
    base = torch.where(torch.isinf(m) & (m < 0), torch.zeros_like(m), m)
    e = torch.exp(z - base)
    total = e.sum(1, keepdim=True)
    lse = (base + torch.log(total))[:, 0]
    empty = torch.isinf(lse) & (lse < 0)
    p = torch.where(empty[:, None], torch.zeros_like(e), e / total)
    log_p = z - base - torch.log(total)  # (a row far from 0 has no digits left for log(total) in lse)
    entropy = torch.where(empty, torch.zeros_like(lse), -torch.where(p == 0, torch.zeros_like(p), p * log_p).sum(1))
    if targets is None:
        return None, lse, entropy, p
    known = (targets >= 0) & (targets < classes)
    at = torch.where(known, targets, 0).long()
    value = log_p.gather(1, at[:, None])[:, 0]
    value = torch.where(empty, torch.full_like(lse, -math.inf), value)
    return torch.where(known, value, torch.zeros_like(lse)), lse, entropy, p


def grad_logits(z, targets, allowed, scale, g_lp=None, g_lse=None, g_h=None):
    n, classes = z.shape
    _, lse, entropy, p = logprobs(z, targets)
    zero = torch.zeros(n, dtype=torch.float64, device=z.device)
    g_lp, g_lse, g_h = (zero if g is None else g.double() for g in (g_lp, g_lse, g_h))
    known = torch.zeros(n, dtype=torch.bool, device=z.device) if targets is None else (targets >= 0) & (targets < classes)
    g_lp = torch.where(known, g_lp, zero)
    at = torch.zeros(n, dtype=torch.int64, device=z.device) if targets is None else torch.where(known, targets, 0).long()
    log_p = torch.where(p == 0, torch.zeros_like(p), torch.log(p.clamp(min=1e-320)))
    grad = p * ((g_lse - g_lp)[:, None] - g_h[:, None] * (log_p + entropy[:, None]))
    grad.scatter_add_(1, at[:, None], g_lp[:, None])
    grad = torch.where((torch.isinf(lse) & (lse < 0))[:, None], torch.zeros_like(grad), grad)
    if allowed is not None:
        grad = torch.where(allowed, grad, torch.zeros_like(grad))
    return grad * scale


def top(logits, allowed, n_top):
    """Classes in the order of the alternatives: larger logits first, NaN before all, the lower class first of equal ones; -1 beyond."""
    x = logits.double().cpu().numpy()
    out = torch.full((x.shape[0], n_top), -1, dtype=torch.int64)
    for r in range(x.shape[0]):
        may = np.arange(x.shape[1]) if allowed is None else np.nonzero(allowed[r].cpu().numpy())[0]
        row = x[r, may]
        nan = np.isnan(row)
        order = may[np.lexsort((may, -np.where(nan, 0.0, row), ~nan))][:n_top]
        out[r, :len(order)] = torch.from_numpy(order)
    return out
