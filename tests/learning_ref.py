"""Plain forms of penalties on logits, of norms and of AdamW steps in 64 bits (PyTorch, any device), and bounds of what arithmetic in 32 bits
may be off by: each rounding is off by U of its result at most."""
import math

import torch

from categorical_ref import EPS, TINY, U, bits

BLOCK = 256


def rounded_bound(value, bound, dtype):
    """`bound` and a rounding to `dtype`."""
    return bound + (value.abs() + bound) * EPS[dtype] * 1.01 + TINY[dtype]


def counts(history, lengths, prompts, n, classes):
    """[n, classes]: how often each class comes in a row's history, how often behind its prompt."""
    device = history.device
    at = torch.arange(history.shape[-1], device=device)
    history = history.long().expand(n, -1)
    most = history.shape[-1]
    lengths = torch.full((n,), most, device=device) if lengths is None else lengths.clamp(0, most)
    prompts = torch.zeros(n, device=device) if prompts is None else prompts.clamp(0, most)
    known = (history >= 0) & (history < classes) & (at < lengths[:, None])
    rows = torch.arange(n, device=device)[:, None] * classes
    count = lambda which: torch.bincount((rows + history)[which], minlength=n * classes).view(n, classes)  # noqa: E731
    return count(known), count(known & (at >= prompts[:, None]))


def _column(x, n, device):
    """A number or each row's, as the kernels have it (32 bits), in 64."""
    x = x.double() if isinstance(x, torch.Tensor) else torch.full((n,), x, device=device).float().double()
    return x.to(device)[:, None]


def penalties(logits, history, lengths=None, prompts=None, repetition=1.0, frequency=0.0, presence=0.0, bias=None, bias_ids=None, bias_values=None,
              allowed=None):
    """(z, bound)"""
    n, classes = logits.shape
    device = logits.device
    x = logits.double()
    if history is None:
        history = torch.zeros(1, 0, dtype=torch.int64, device=device)
    seen, said = counts(history, lengths, prompts, n, classes)
    r, f, q = (_column(v, n, device) for v in (repetition, frequency, presence))
    z = torch.where(seen > 0, torch.where(x > 0, x / r, x * r), x)
    bound = torch.where(seen > 0, 2.01 * z.abs() * U, 0.0)  # (a product with 1 / r, which is rounded, too)
    less = f * said + q
    bound = bound + torch.where(said > 0, U * ((f * said).abs() + 2 * less.abs()), 0.0)  # (product, sum, and the sum's own error)
    z = torch.where(said > 0, z - less, z)
    bound = bound + torch.where(said > 0, U * z.abs(), 0.0)
    if bias is not None:
        z = z + bias.double()
        bound = bound + U * z.abs()
    if bias_ids is not None:
        known = (bias_ids >= 0) & (bias_ids < classes)
        rows = torch.arange(n, device=device)[:, None] * classes
        at = (rows + bias_ids.long())[known]
        add = lambda v: torch.zeros(n * classes, dtype=torch.float64, device=device).index_add_(0, at, v).view(n, classes)  # noqa: E731
        many = add(torch.ones(len(at), dtype=torch.float64, device=device))
        values = bias_values.double()[known]
        z = z + add(values)
        bound = bound + torch.where(many > 0, U * (many - 1).clamp(min=0) * add(values.abs()) + U * z.abs(), 0.0)
    bound = rounded_bound(z, bound * 1.01, logits.dtype)
    # beyond the largest number of a type, and half a step more, there is only infinity: twice float32's lowest value is one
    z = torch.where(z.abs() >= torch.finfo(logits.dtype).max * (1 + EPS[logits.dtype] / 2), z * math.inf, z)
    if allowed is not None:
        z = torch.where(bits(allowed, classes), z, -math.inf)
    return z, bound


def penalties_grad(grad, logits, history, lengths=None, repetition=1.0, allowed=None):
    """(gradient of the logits, bound, gradient of a shared bias, bound)"""
    n, classes = logits.shape
    g = grad.double()
    if allowed is not None:
        g = torch.where(bits(allowed, classes), g, 0.0)
    if history is None:
        history = torch.zeros(1, 0, dtype=torch.int64, device=logits.device)
    seen, _ = counts(history, lengths, None, n, classes)
    r = _column(repetition, n, logits.device)
    dx = torch.where(seen > 0, torch.where(logits.double() > 0, g / r, g * r), g)
    if allowed is not None:
        dx = torch.where(bits(allowed, classes), dx, 0.0)
    bias = g.sum(0)
    return dx, rounded_bound(dx, 2 * U * dx.abs(), grad.dtype), bias, n * U * g.abs().sum(0) + TINY[torch.float32]


def close(got, want, bound):
    """Whether all values are within their bounds; what is not finite has to be the same."""
    got = got.double()
    finite = torch.isfinite(want)
    same = torch.where(torch.isnan(want), torch.isnan(got), got == want)
    return bool(torch.where(finite, (got - want).abs() <= bound, same).all())


# ---- AdamW --------------------------------------------------------------------------------------------------------------

def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 (Salmon et al., 2011) of int64 tensors or numbers of 32 bits."""
    def times(a, m):
        low, high = (a & 0xffff) * m, (a >> 16) * m
        high = high + (low >> 16)
        return high >> 16, ((high & 0xffff) << 16) | (low & 0xffff)

    k0, k1 = seed & 0xffffffff, seed >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = times(c0, 0xD2511F53), times(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return c0, c1, c2, c3


def words(n, seed, step, tensor, device):
    """The random bits of a tensor's n numbers, as the header says."""
    quad = torch.arange((n + 3) // 4, device=device)
    w = philox(quad & 0xffffffff, (quad >> 32 << 8) + 6, torch.full_like(quad, step & 0xffffffff), torch.full_like(quad, tensor), seed)
    return torch.stack(w, 1).view(-1)[:n]


def m_values(code, scale):
    """Numbers of 8-bit codes (1-d) and their blocks' scales."""
    c = code.double()
    return torch.where(code == -128, math.nan, c * c.abs()) * scale.double().repeat_interleave(BLOCK)[:len(c)]


def v_values(code, scale):
    c = code.double()
    return torch.where(code == 255, math.nan, (c * c * scale.double().repeat_interleave(BLOCK)[:len(c)]) ** 2)


def block_max(x):
    x = torch.where(torch.isfinite(x), x.abs(), 0.0)
    pad = torch.zeros(-len(x) % BLOCK, dtype=x.dtype, device=x.device)
    return torch.cat([x, pad]).view(-1, BLOCK).amax(1)


def m_codes(level, u):
    """Codes of levels (sqrt of what is in units of the scale), rising in them."""
    c = level.floor().clamp(max=126)
    return c + (level ** 2 - c ** 2 > (2 * c + 1) * u).double()


def v_codes(level, u):
    c = level.floor().clamp(max=253)
    c = c + (level ** 4 - c ** 4 > ((c + 1) ** 4 - c ** 4) * u).double()
    return torch.where(level > 0, c.clamp(min=1), c)


def adamw(p, g, m, v, *, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, scale=1.0, factor=1.0):
    """New (p, m, v) in 64 bits and their bounds, all 1-d.  m and v: 64 bits."""
    b1, b2 = betas
    p, x = p.double(), g.double() * (scale * factor)
    new_m = b1 * m + (1 - b1) * x
    m_bound = U * (2.5 * (b1 * m).abs() + 4.5 * ((1 - b1) * x).abs() + new_m.abs()) * 1.01
    new_v = b2 * v + (1 - b2) * x * x
    v_bound = U * (2.5 * b2 * v + 7.5 * (1 - b2) * x * x + new_v) * 1.01
    root = torch.sqrt(new_v)
    denominator = root / math.sqrt(1 - b2 ** step) + eps
    size = lr / (1 - b1 ** step)
    update = size * new_m / denominator
    update = torch.where(new_m == 0, torch.zeros_like(update) if eps > 0 else update, update)
    new_p = p * (1 - lr * weight_decay) - update
    v_off = torch.where(new_v > 0, v_bound / new_v.clamp(min=1e-300), 0.0)
    p_bound = (U * (2.5 * p.abs() + new_p.abs()) + update.abs() * (12 * U + v_off) + abs(size) * m_bound / denominator.clamp(min=1e-300)) * 1.01
    tiny = 2.0 ** -140  # (sums of products that have fewer places than 24)
    return new_p, p_bound + tiny, new_m, m_bound + tiny, new_v, v_bound + tiny


def rounded_at_random(x, word):
    """To bfloat16, of 64-bit numbers: what the 12 bits and a half make of them (rising in x)."""
    f = x.float()
    sums = f.view(torch.int32).long() + ((word >> 20 << 4) | 8)
    return torch.where(torch.isfinite(f), (sums & ~0xffff).to(torch.int32).view(torch.float32), f).double()
