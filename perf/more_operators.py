"""What a categorical model learns with and answers through, as cases that can be timed and compared.

A model that has been given log densities and gradients (perf/operators.py) learns by steps over all of its parameters: the
gradients' common norm (`norm`), which bounds the step, and AdamW steps over many tensors at once, with moments of 32 bits
(`adamw`) or of 8 (`adamw8`).  Before it answers, its logits are adjusted: classes that were said before are penalised, biases are added, what a
grammar rules out becomes -infinity (`penalties`), and a model that is trained through that needs its gradient (`penalties_grad`).

`run` computes one of these: where `own` is false from elementary torch operations in 32 bits (sums of squares in 64), rounded once at the
end, otherwise by the framework's operators.  `listed()` are fixed cases over the range; `draw(rng)` gives further ones of
the same ranges.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
IDS = {"i32": torch.int32, "i64": torch.int64}
BLOCK = 256  # elements of a tensor that share the scales of their 8-bit moments


def _logits(name, op, dtype, n, classes, history, *, pad=0, shared=False, prompt=0.0, mask="", bias=False, n_bias=0, in_place=False, ids="i64"):
    """n rows of logits, `classes` + pad numbers apart, with up to `history` classes said before each (shared: one text, of which row i
    has seen the beginning), a part `prompt` of them not by the model.  mask: "rows" rules out a quarter of the classes row by row, "one"
    for all rows alike.  bias: one for each class.  n_bias: biases of single classes, row by row."""
    return {"name": name, "op": op, "dtype": dtype, "n": n, "classes": classes, "history": history, "pad": pad, "shared": shared,
            "prompt": prompt, "mask": mask, "bias": bias, "n_bias": n_bias, "in_place": in_place, "ids": ids}


def _step(name, op, tensors, total, params, grads, *, copy="", clip=False, decay=0.01, step=1000):
    """`tensors` tensors of `total` elements together, of which the largest has up to a thousand times the smallest's."""
    return {"name": name, "op": op, "tensors": tensors, "total": total, "params": params, "grads": grads, "copy": copy, "clip": clip,
            "decay": decay, "step": step}


def listed():
    return [
        # a decoding step of 8 sequences, adjusted where the logits are: latency
        _logits("penalties, 8 rows, in place", "penalties", "bf16", 8, 32000, 512, prompt=0.25, in_place=True),
        # a decoding step of 64 long conversations whose next word a grammar and the caller's biases have a say in
        _logits("penalties, 64 rows", "penalties", "bf16", 64, 128000, 4096, prompt=0.75, mask="rows", n_bias=32),
        # every place of a text of 4096 tokens, as it was answered: what was said before it, with a bias of each class
        _logits("penalties, 4096 rows", "penalties", "bf16", 4096, 32001, 4096, pad=63, shared=True, bias=True, ids="i32"),
        # a regression on 1000 observations of one of 1000 classes, with an intercept for each class
        _logits("penalties_grad, 1000 rows of 1000", "penalties_grad", "f32", 1000, 1000, 10, bias=True, ids="i32"),
        # a policy's gradient through what its answers of 4096 tokens were adjusted with
        _logits("penalties_grad, 4096 rows", "penalties_grad", "bf16", 4096, 50001, 4096, pad=7, shared=True, prompt=0.25, mask="one", bias=True),
        # the word model of 1000 words with 8 features: latency
        _step("norm, 2 tensors", "norm", 2, 16000, "f32", "f32"),
        # all gradients of a model of 200 million parameters
        _step("norm, 150 tensors", "norm", 150, 200_000_000, "bf16", "bf16"),
        # the word model's step
        _step("adamw, 2 tensors", "adamw", 2, 16000, "f32", "f32", step=1),
        # the step of a model of 120 million parameters that is computed in 16 bits, bounded by the gradients' norm
        _step("adamw, 150 tensors", "adamw", 150, 120_000_000, "f32", "bf16", copy="bf16", clip=True),
        # a table of 100003 rows of 1024, all in 32 bits
        _step("adamw, a table", "adamw", 1, 100003 * 1024, "f32", "f32", decay=0.0),
        # a small model in 16 bits throughout
        _step("adamw8, 20 tensors", "adamw8", 20, 1_500_000, "bf16", "bf16", step=10),
        # a model of 200 million parameters whose moments are to leave room for its activations
        _step("adamw8, 150 tensors", "adamw8", 150, 200_000_000, "f32", "bf16", copy="bf16"),
    ]


def _between(rng, low, high):
    """A whole number, its logarithm spread evenly."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["penalties", "penalties", "penalties_grad", "norm", "adamw", "adamw8"])
    if op in ("penalties", "penalties_grad"):
        dtype = rng.choice(["bf16", "f16", "f32"])
        while True:
            n, classes, history = _between(rng, 1, 4096), _between(rng, 1000, 160000), _between(rng, 1, 16384)
            if n * classes * SIZES[dtype] <= 4096 * 32001 * 2 and n * history <= 1 << 23:
                break
        mask, bias = rng.choice(["", "", "rows", "one"]), rng.random() < 0.5
        case = _logits("", op, dtype, n, classes, history, pad=rng.choice([0, 0, 1, 13, 64, 96]), shared=rng.random() < 0.3,
                       prompt=rng.choice([0.0, round(rng.random(), 3)]), mask=mask, bias=bias,
                       n_bias=rng.choice([0, 0, 1, 300, rng.randrange(2, 100)]) if op == "penalties" else 0,
                       in_place=op == "penalties" and rng.random() < 0.4, ids=rng.choice(["i32", "i64"]))
    else:
        tensors, total = _between(rng, 1, 300), _between(rng, 1000, 120_000_000)
        grads = rng.choice(["f32", "bf16", "bf16", "f16"])
        params = grads if op == "norm" else rng.choice(["f32", "f32", "bf16"])
        case = _step("", op, tensors, total, params, grads, copy=rng.choice(["", "bf16", "f16"]) if params == "f32" and op != "norm" else "",
                     clip=op != "norm" and rng.random() < 0.3, decay=rng.choice([0.0, 0.01, 0.1]), step=_between(rng, 1, 100000))
    del case["name"]
    return case


# ---- what a program has in hand ---------------------------------------------------------------------------------------

# How often a class comes: class v of V with probability ((v + 1) / V)^(1/4) - (v / V)^(1/4), so that a few are said again
# and again and most never; then the classes change places.

def _classes(classes, shape, gen):
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    v = (u ** 4 * classes).long().clamp_(max=classes - 1)
    step = 7919
    while math.gcd(step, classes) != 1:
        step += 2
    return v * step % classes


def _seen(case):
    """Different classes in a row's history, on average, and of those that are biased, too."""
    v = torch.arange(case["classes"] + 1, dtype=torch.float64)
    p = torch.diff((v / case["classes"]) ** 0.25).clamp(max=1 - 1e-12)
    mean = 0.0
    for part in range(8):  # (lengths are spread evenly)
        mean += float((1.0 - torch.exp(case["history"] * (part + 0.5) / 8 * torch.log1p(-p))).sum()) / 8
    return mean


def _prepare_logits(case, gen):
    dtype, n, classes, length = DTYPES[case["dtype"]], case["n"], case["classes"], case["history"]
    s = dict(case)
    uniform = lambda low, high: torch.rand(n, generator=gen, device="cuda") * (high - low) + low  # noqa: E731
    s["logits"] = (torch.randn(n, classes + case["pad"], generator=gen, device="cuda") * 3.0).to(dtype)[:, :classes]
    history = _classes(classes, (1 if case["shared"] else n, length), gen)
    # one place in sixteen is padding
    history = torch.where(torch.rand(history.shape, generator=gen, device="cuda") < 1 / 16, -1, history)
    s["history"] = history.to(IDS[case["ids"]])
    if case["shared"]:
        s["lengths"] = (torch.arange(n, device="cuda") * length // n).int()
    else:
        s["lengths"] = torch.randint(0, length + 1, (n,), generator=gen, device="cuda").int()
    s["prompts"] = (s["lengths"] * case["prompt"]).int() if case["prompt"] else None
    s["repetition"], s["frequency"], s["presence"] = uniform(1.0, 1.5), uniform(0.0, 0.5), uniform(-0.5, 1.0)
    s["allowed"] = s["dense_bias"] = s["bias_ids"] = s["bias_values"] = None
    if case["mask"]:
        shape = (n if case["mask"] == "rows" else 1, (classes + 31) // 32)
        words = lambda: torch.randint(-2**31, 2**31, shape, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)  # noqa: E731
        s["allowed"] = words() | words()  # bit v % 32 of word v / 32: class v is allowed
        if case["mask"] == "one":
            s["allowed"] = s["allowed"][0]
    if case["bias"]:
        s["dense_bias"] = torch.randn(classes, generator=gen, device="cuda")
    if case["n_bias"]:
        s["bias_ids"] = _classes(classes, (n, case["n_bias"]), gen).to(IDS[case["ids"]])
        s["bias_values"] = torch.randn(n, case["n_bias"], generator=gen, device="cuda") * 4.0
    if case["op"] == "penalties_grad":
        s["grad"] = (torch.randn(n, classes + case["pad"], generator=gen, device="cuda") / n).to(dtype)[:, :classes]
    return s


def _sizes(case):
    r = random.Random(case["tensors"] * 1000003 + case["total"])
    share = [math.exp(r.uniform(0.0, math.log(1000.0))) for _ in range(case["tensors"])]
    return [max(1, int(case["total"] * w / sum(share))) for w in share]


def _prepare_tensors(case, gen):
    """Tensors that lie one behind the other, each from the beginning of a block on; between them there are zeros."""
    s = dict(case)
    sizes = _sizes(case)
    first, size_of = [], []
    blocks = 0
    for size in sizes:
        first.append(blocks)
        size_of.append((size + BLOCK - 1) // BLOCK)
        blocks += size_of[-1]
    n = blocks * BLOCK
    s["sizes"] = sizes
    # of each block: its tensor, and its place there; of each element: whether there is one
    s["tensor"] = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(size_of, device="cuda"))
    s["place"] = torch.arange(blocks, device="cuda") - torch.tensor(first, device="cuda")[s["tensor"]]
    end = torch.tensor(sizes, device="cuda")[s["tensor"]]
    there = s["place"][:, None] * BLOCK + torch.arange(BLOCK, device="cuda") < end[:, None]
    # each tensor's gradients have a size of their own
    spread = torch.exp(torch.randn(len(sizes), generator=gen, device="cuda") - 7.0)[s["tensor"]][:, None]

    def normal(scale, dtype=torch.float32):
        return (torch.randn(blocks, BLOCK, generator=gen, device="cuda").mul_(scale).mul_(there)).to(dtype).view(-1)

    def views(flat, each=1):
        return [flat[b * BLOCK // each:b * BLOCK // each + (k if each == 1 else c)] for b, k, c in zip(first, sizes, size_of)]

    s["grad"] = normal(spread, DTYPES[case["grads"]])
    s["grads_of"] = views(s["grad"])
    if case["op"] == "norm":
        return s
    s["param"] = normal(0.02, DTYPES[case["params"]])
    s["params_of"] = views(s["param"])
    s["copies"] = torch.zeros(n, dtype=DTYPES[case["copy"]], device="cuda") if case["copy"] else None
    if case["op"] == "adamw":
        s["m"] = normal(spread * 0.3)
        s["v"] = normal(spread).square_()
        states = views(s["m"]), views(s["v"])
    else:
        # codes as steps leave them: most far below their block's largest, which has the last one
        code = lambda last, floor: (torch.rand(blocks, BLOCK, generator=gen, device="cuda") ** 2 * last).clamp_(floor).floor_()  # noqa: E731
        m, v = code(128, 0).clamp_(max=127), code(255, 1).clamp_(max=254)
        m[:, 0], v[:, 0] = 127, 254
        m *= torch.randint(0, 2, m.shape, generator=gen, device="cuda") * 2 - 1
        s["m"] = (m * there).to(torch.int8).view(-1)
        s["v"] = (v * there).to(torch.uint8).view(-1)
        del m, v
        size = spread[:, 0] * (1.0 + torch.rand(blocks, generator=gen, device="cuda"))
        s["m_scale"], s["v_scale"] = size / 127.0 ** 2, 2.0 * size / 254.0 ** 2
        s["m_value"], s["v_value"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        s["values_of"] = views(s["m_value"]), views(s["v_value"])
        states = views(s["m"]), views(s["v"]), views(s["m_scale"], BLOCK), views(s["v_scale"], BLOCK)
    if own:  # the handle that a training program keeps
        import paper_1910_11141_amd as nuts

        s["moments"] = nuts.Moments(s["params_of"], bits=32 if case["op"] == "adamw" else 8, states=states,
                                    copies=views(s["copies"]) if case["copy"] else None)
    return s


LR, BETA1, BETA2, EPS, MAX_NORM, SEED = 1e-3, 0.9, 0.999, 1e-8, 1.0, 20


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_logits if "classes" in case else _prepare_tensors)(case, gen)


# ---- the framework's calls ----------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_1910_11141_amd as nuts

    if s["op"] == "penalties":
        return nuts.nuts_penalties(s["logits"], s["history"], lengths=s["lengths"], prompts=s["prompts"], repetition=s["repetition"],
                                   frequency=s["frequency"], presence=s["presence"], bias=s["dense_bias"], bias_ids=s["bias_ids"],
                                   bias_values=s["bias_values"], allowed=s["allowed"], out=s["logits"] if s["in_place"] else None)
    if s["op"] == "penalties_grad":
        grad, bias = nuts.nuts_penalties_grad(s["grad"], s["logits"], s["history"], lengths=s["lengths"], repetition=s["repetition"],
                                              allowed=s["allowed"], want_bias=s["bias"])
        return {"grad": grad, "bias": bias}
    if s["op"] == "norm":
        got = nuts.nuts_norm(s["grads_of"], max_norm=MAX_NORM)
        return {"norm": got.norm, "factor": got.factor}
    out = {}
    factor = None
    if s["clip"]:
        out["norm"], factor = nuts.nuts_norm(s["grads_of"], max_norm=MAX_NORM)
    nuts.nuts_adamw(s["moments"], s["grads_of"], step=s["step"], lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=s["decay"], factor=factor, seed=SEED)
    if s["op"] == "adamw8":
        nuts.nuts_adamw_values(s["moments"], out=s["values_of"])
    return out | _state(s)


def _state(s):
    if s["op"] == "adamw":
        return {"param": s["param"], "copy": s["copies"], "m": s["m"], "v": s["v"]}
    return {"param": s["param"], "copy": s["copies"], "m": s["m_value"], "v": s["v_value"]}


# ---- plain forms --------------------------------------------------------------------------------------------------------

def _counts(s):
    """(how often each class comes in each row's history, how often behind its prompt)"""
    n, classes, history = s["n"], s["classes"], s["history"].long()
    at = torch.arange(s["history"].shape[1], device="cuda")
    known = (history >= 0) & (history < classes) & (at < s["lengths"][:, None])
    history = torch.where(known, history, classes)
    ones = torch.ones(history.shape, device="cuda")
    seen = torch.zeros(n, classes + 1, device="cuda").scatter_add_(1, history, ones)[:, :classes]
    if s["prompts"] is None:
        return seen, seen
    said = torch.zeros(n, classes + 1, device="cuda").scatter_add_(1, history, (at >= s["prompts"][:, None]).float())[:, :classes]
    return seen, said


def _ruled_out(s):
    v = torch.arange(s["classes"], device="cuda")
    return (s["allowed"][..., v >> 5] >> (v & 31)) & 1 == 0


def _penalties(s):
    z = s["logits"].float()
    seen, said = _counts(s)
    r = s["repetition"][:, None]
    z = torch.where(seen > 0, torch.where(z > 0, z / r, z * r), z)
    z = z - (s["frequency"][:, None] * said + s["presence"][:, None] * (said > 0))
    if s["dense_bias"] is not None:
        z = z + s["dense_bias"]
    if s["bias_ids"] is not None:
        z = z.scatter_add(1, s["bias_ids"].long(), s["bias_values"])
    if s["allowed"] is not None:
        z = z.masked_fill(_ruled_out(s), -math.inf)
    z = z.to(s["logits"].dtype)
    return s["logits"].copy_(z) if s["in_place"] else z


def _penalties_grad(s):
    z, grad, r = s["logits"].float(), s["grad"].float(), s["repetition"][:, None]
    if s["allowed"] is not None:
        grad = grad.masked_fill(_ruled_out(s), 0.0)
    seen, _ = _counts(s)
    factor = torch.where(seen > 0, torch.where(z > 0, 1.0 / r, r), 1.0)
    return {"grad": (grad * factor).to(s["logits"].dtype), "bias": grad.sum(dim=0) if s["bias"] else None}


def _norm(s):
    norm = s["grad"].double().square().sum().sqrt()
    return {"norm": norm.float(), "factor": (MAX_NORM / norm).clamp(max=1.0).float()}


def _times(a, by):
    """High and low 32 bits of the product of whole numbers of 32 bits."""
    low, high = (a & 0xffff) * by, (a >> 16) * by
    high = high + (low >> 16)
    return high >> 16, (high & 0xffff) << 16 | (low & 0xffff)


def _words(s):
    """32 random bits for each element: Philox4x32-10 with key SEED, one counter for four elements of a tensor."""
    quad = s["place"][:, None] * (BLOCK // 4) + torch.arange(BLOCK // 4, device="cuda")
    c0, c1 = quad & 0xffffffff, (quad >> 32) << 8 | 6
    c2, c3 = torch.full_like(quad, s["step"]), s["tensor"][:, None].expand_as(quad)
    k0, k1 = SEED & 0xffffffff, SEED >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = _times(c0, 0xD2511F53), _times(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return torch.stack([c0, c1, c2, c3], dim=2).view(-1, BLOCK)


def _adamw(s):
    out = _norm(s) if s["clip"] else {}
    g = s["grad"].float()
    if s["clip"]:
        g = g * out.pop("factor")
    eight, low = s["op"] == "adamw8", s["param"].dtype == torch.bfloat16
    words = _words(s) if eight or low else None
    if eight:
        code = s["m"].view(-1, BLOCK).float()
        m = (torch.sign(code) * code * code * s["m_scale"][:, None]).view(-1)
        code = s["v"].view(-1, BLOCK).float()
        v = (code * code * s["v_scale"][:, None]).square().view(-1)
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    root = torch.sqrt(v)
    p = s["param"].float() * (1.0 - LR * s["decay"])
    p = p - (LR / (1.0 - BETA1 ** s["step"])) * m / (root * (1.0 / math.sqrt(1.0 - BETA2 ** s["step"])) + EPS)
    if low:
        # up or down with the probabilities that keep the mean: 12 bits of chance above the 16 that go
        bits = p.view(torch.int32).long() + ((words >> 20) << 4 | 8).view(-1)
        p = (bits & ~0xffff).to(torch.int32).view(torch.float32)
    s["param"].copy_(p)
    if s["copies"] is not None:
        s["copies"].copy_(p)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        m, root = m.view(-1, BLOCK), root.view(-1, BLOCK)
        scale = m.abs().amax(dim=1) * (1.0 / 127.0 ** 2)
        x = torch.where(scale[:, None] > 0, m.abs() / scale[:, None], 0.0)
        code = torch.floor(torch.sqrt(x)).clamp(max=126.0)
        code = code + (x - code * code > (2.0 * code + 1.0) * (((words & 1023) + 0.5) * (1.0 / 1024.0)).float())
        code = torch.where(m < 0, -code, code)
        s["m"].view(-1, BLOCK).copy_(code)
        s["m_scale"].copy_(scale)
        s["m_value"].view(-1, BLOCK).copy_(torch.sign(code) * code * code * scale[:, None])
        scale = root.amax(dim=1) * (1.0 / 254.0 ** 2)
        x = torch.where(scale[:, None] > 0, root / scale[:, None], 0.0)
        code = torch.floor(torch.sqrt(x)).clamp(max=253.0)
        below, above = code * code, (code + 1.0) * (code + 1.0)
        code = code + (x * x - below * below > (above - below) * (above + below) * (((words >> 10 & 1023) + 0.5) * (1.0 / 1024.0)).float())
        code = torch.where(root > 0, code.clamp(min=1.0), code)
        s["v"].view(-1, BLOCK).copy_(code)
        s["v_scale"].copy_(scale)
        s["v_value"].view(-1, BLOCK).copy_((code * code * scale[:, None]).square())
    return out | _state(s)


def run(s):
    if own:
        return _run_own(s)
    return {"penalties": _penalties, "penalties_grad": _penalties_grad, "norm": _norm}.get(s["op"], _adamw)(s)


# ---- 64 bits ------------------------------------------------------------------------------------------------------------

def _exact_logits(s):
    """Row by row counts from each history's distinct classes; logits as they follow from them in 64 bits."""
    n, classes, rows = s["n"], s["classes"], torch.arange(s["n"], device="cuda")[:, None]
    history = s["history"].long().expand(n, -1)
    place = torch.arange(history.shape[1], device="cuda")[None, :]
    some = (history >= 0) & (place < s["lengths"][:, None])
    flat = (rows * classes + history)[some]
    seen = torch.bincount(flat, minlength=n * classes).view(n, classes)
    said = seen
    if s["prompts"] is not None:
        flat = (rows * classes + history)[some & (place >= s["prompts"][:, None])]
        said = torch.bincount(flat, minlength=n * classes).view(n, classes)
    x, r = s["logits"].double(), s["repetition"].double()[:, None]
    slope = torch.where(seen == 0, 1.0, torch.where(x > 0, 1 / r, r))
    may = None
    if s["allowed"] is not None:
        bits = s["allowed"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32) & 1
        may = bits.flatten(-2)[..., :classes].bool()
    if s["op"] == "penalties_grad":
        g = s["grad"].double()
        if may is not None:
            g = torch.where(may, g, 0.0)
        return {"grad": g * slope, "bias": g.sum(0) if s["bias"] else None}
    z = x * slope - s["frequency"].double()[:, None] * said - s["presence"].double()[:, None] * (said > 0).double()
    if s["dense_bias"] is not None:
        z += s["dense_bias"].double()[None, :]
    if s["bias_ids"] is not None:
        z.view(-1).index_add_(0, (rows * classes + s["bias_ids"].long()).view(-1), s["bias_values"].double().view(-1))
    return z if may is None else torch.where(may, z, -math.inf)


def exact(case, seed):
    """What `run` returns for these inputs, in 64 bits; the random bits are as given there."""
    s = prepare(case, seed)
    if "classes" in s:
        return _exact_logits(s)
    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g)
    factor = min(1.0, MAX_NORM / float(norm))
    if s["op"] == "norm":
        return {"norm": norm, "factor": torch.tensor(factor, dtype=torch.float64)}
    eight, t = s["op"] == "adamw8", s["step"]
    if s["clip"]:
        g *= factor
    if eight:
        c = s["m"].double().view(-1, BLOCK)
        m = (c * c.abs() * s["m_scale"].double()[:, None]).view(-1)
        v = (s["v"].double().view(-1, BLOCK) ** 4 * s["v_scale"].double()[:, None] ** 2).view(-1)
    else:
        m, v = s["m"].double(), s["v"].double()
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    p = s["param"].double()
    p = p - LR * (s["decay"] * p + m / -math.expm1(t * math.log(BETA1)) / (torch.sqrt(v / -math.expm1(t * math.log(BETA2))) + EPS))
    low = s["param"].dtype == torch.bfloat16
    out = {"norm": norm} if s["clip"] else {}
    # (a parameter of 16 bits, rounded at random, has a mean that is not rounded and no other value in 64 bits)
    out |= {"param": None if low else p, "copy": p if s["copies"] is not None else None}
    if not eight:
        return out | {"m": m, "v": v}
    # the same for moments: their places in the row of values that 8 bits stand for are the random bits'
    words = _words(s)
    top = m.abs().view(-1, BLOCK).amax(1, keepdim=True).clamp(min=1e-300)
    level = torch.sqrt(m.abs().view(-1, BLOCK) / top) * 127.0
    low_end = level.floor().clamp(max=126.0)
    share = (level ** 2 - low_end ** 2) / (2 * low_end + 1)
    code = low_end + (share > ((words & 1023) + 0.5) / 1024.0).double()
    m_value = torch.sign(m) * (code ** 2 * top / 127.0 ** 2).view(-1)
    top = v.view(-1, BLOCK).amax(1, keepdim=True).clamp(min=1e-300)
    level = (v.view(-1, BLOCK) / top) ** 0.25 * 254.0
    low_end = level.floor().clamp(max=253.0)
    share = (level ** 4 - low_end ** 4) / ((low_end + 1) ** 4 - low_end ** 4)
    code = low_end + (share > ((words >> 10 & 1023) + 0.5) / 1024.0).double()
    code = torch.where(v.view(-1, BLOCK) > 0, code.clamp(min=1.0), 0.0)
    return out | {"m": m_value, "v": (code ** 4 * top / 254.0 ** 4).view(-1)}


# ---- what cannot be done without ----------------------------------------------------------------------------------------

def work(case):
    if "classes" in case:
        n, classes, size, id_bytes = case["n"], case["classes"], SIZES[case["dtype"]], 4 if case["ids"] == "i32" else 8
        mask = {"": 0, "rows": n, "one": 1}[case["mask"]] * ((classes + 31) // 32) * 4
        history = (1.0 if case["shared"] else n / 2) * case["history"] * id_bytes  # (rows of half of it, on average)
        seen = n * _seen(case)
        more = mask + history + n * 20 + (4 * classes if case["bias"] else 0) + n * case["n_bias"] * (4 + id_bytes)
        said = (0.5 if case["shared"] else n / 2) * case["history"]
        if case["op"] == "penalties_grad":
            return {"bytes": 2 * n * classes * size + seen * size + more, "flops": n * classes * (1 if case["bias"] else 0) + 2 * seen + said}
        if case["in_place"] and not case["bias"]:
            # what is neither said, biased nor ruled out stays as it is
            touched = seen + n * case["n_bias"]
            return {"bytes": 2 * size * touched + (n * classes * size / 4 if case["mask"] else 0) + more, "flops": 4 * touched + said}
        return {"bytes": 2 * n * classes * size + more, "flops": n * classes * (1 if case["bias"] else 0) + 4 * seen + said}
    n, grad = sum(_sizes(case)), SIZES[case["grads"]]
    if case["op"] == "norm":
        return {"bytes": n * grad, "flops": 2 * n}
    each = 2 * SIZES[case["params"]] + SIZES[case["copy"]] + grad * (2 if case["clip"] else 1)
    # 8 bits: codes are read and written, and read again for the values in 16 bits that are returned
    each += 16 if case["op"] == "adamw" else 6 + 4 + 24 / BLOCK
    return {"bytes": n * each, "flops": n * ((16 if case["op"] == "adamw" else 40) + (3 if case["clip"] else 0))}
