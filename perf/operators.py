"""The categorical operators' work, as cases that can be timed and compared.

A categorical model draws each of its observations from one of many classes - the next token of a text, one word of a
vocabulary - and what it does with them is: look up the rows of a table that belong to a batch of classes (`lookup`), add
the gradients of such rows up class by class (`lookup_grad`), say how probable given classes are under a row of logits,
with the row's entropy and its most probable classes (`logprobs`), differentiate that (`logprobs_grad`), and do the same
from the features and the class weights, whose products the logits are (`score`, `score_grad`).

`run` computes one of these: where `own` is false from elementary torch operations in 32 bits, rounded once at the end,
otherwise by the framework's operators.  `listed()` are fixed cases over the range; `draw(rng)` gives further ones of the same
ranges.  A gradient's case is a training step's share: the forward pass, whose statistics the gradient needs, and the gradient.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
IDS = {"i32": torch.int32, "i64": torch.int64}
IGNORED = -100   # a target outside the classes: the row has none


def _lookup(name, op, dtype, n, classes, dim, *, scale=1.0, ids="i64"):
    """n rows of a table of `classes` rows of `dim` numbers; some classes are far more frequent than others."""
    return {"name": name, "op": op, "dtype": dtype, "n": n, "classes": classes, "dim": dim, "scale": scale, "ids": ids}


def _logits(name, op, dtype, n, classes, *, pad=0, top=0, mask=False, scale=1.0, ids="i64", entropy=False):
    """n rows of logits that are `classes` + pad numbers apart.  mask: a part of the classes is ruled out, row by row.
    entropy: the entropy has a gradient, too."""
    return {"name": name, "op": op, "dtype": dtype, "n": n, "classes": classes, "pad": pad, "top": top, "mask": mask,
            "scale": scale, "ids": ids, "entropy": entropy}


def _score(name, op, dtype, n, classes, dim, *, scale=1.0, ids="i64"):
    """n feature vectors of `dim` numbers against the weights of `classes` classes."""
    return {"name": name, "op": op, "dtype": dtype, "n": n, "classes": classes, "dim": dim, "scale": scale, "ids": ids}


def listed():
    return [
        # a decoding step of 64 sequences: latency
        _lookup("lookup, 64 tokens", "lookup", "bf16", 64, 32000, 1024, scale=32.0),
        # a training batch of 16 sequences of 4096 tokens
        _lookup("lookup, 65536 tokens", "lookup", "bf16", 65536, 100003, 2048, scale=math.sqrt(2048)),
        # group effects of a regression: 1000 observations of 100 features each, binary32
        _lookup("lookup_grad, 1000 rows of 100", "lookup_grad", "f32", 1000, 5000, 100, scale=0.5, ids="i32"),
        # the training batch's gradient
        _lookup("lookup_grad, 65536 tokens", "lookup_grad", "bf16", 65536, 100003, 2048, scale=math.sqrt(2048)),
        # a decoding step of 8 sequences that may only go on with part of the vocabulary: alternatives to choose from
        _logits("logprobs, 8 rows, 20 alternatives", "logprobs", "bf16", 8, 128000, top=20, mask=True, scale=1.25),
        # the log-probabilities of a prompt of 4096 tokens with the five most probable ones of each place
        _logits("logprobs, 4096 rows", "logprobs", "bf16", 4096, 32001, pad=63, top=5),
        # a regression on 1000 observations of one of 1000 classes
        _logits("logprobs_grad, 1000 rows of 1000", "logprobs_grad", "f32", 1000, 1000, ids="i32"),
        # the loss of a policy with an entropy bonus on 4096 tokens
        _logits("logprobs_grad, 4096 rows", "logprobs_grad", "bf16", 4096, 50001, pad=7, entropy=True),
        # the regression of 1000 observations of 25 features, with 1000 classes in place of two
        _score("score, 1000 rows of 25", "score", "f32", 1000, 1000, 25, ids="i32"),
        # the log-probabilities of 8192 tokens of a text
        _score("score, 8192 rows of 4096", "score", "bf16", 8192, 32000, 4096),
        # the regression of 10000 observations of 100 features, with 1000 classes in place of two
        _score("score_grad, 10000 rows of 100", "score_grad", "f32", 10000, 1000, 100, ids="i32"),
        # a training step's loss on 4096 tokens
        _score("score_grad, 4096 rows of 2048", "score_grad", "bf16", 4096, 32001, 2048),
    ]


def _between(rng, low, high):
    """A whole number, its logarithm spread evenly."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "logprobs", "logprobs_grad", "score", "score_grad"])
    ids = rng.choice(["i32", "i64"])
    if op in ("lookup", "lookup_grad"):
        dtype = rng.choice(["bf16", "f16", "f32"])
        while True:
            n, classes, dim = _between(rng, 1, 65536), _between(rng, 1000, 160000), _between(rng, 25, 4096)
            if rng.random() < 0.5:
                dim = max(32, dim // 32 * 32) + (32 if dim // 32 == 96 else 0)
            if max(n, classes) * dim * SIZES[dtype] <= 100003 * 2048 * 2:
                break
        case = _lookup("", op, dtype, n, classes, dim, scale=rng.choice([1.0, round(rng.uniform(0.25, 64.0), 3)]), ids=ids)
    elif op in ("logprobs", "logprobs_grad"):
        dtype = rng.choice(["bf16", "f16", "f32"])
        while True:
            n, classes = _between(rng, 1, 8192), _between(rng, 1000, 160000)
            if n * classes * SIZES[dtype] <= 4096 * 32001 * 2:
                break
        mask = rng.random() < 0.4
        case = _logits("", op, dtype, n, classes, pad=rng.choice([0, 0, 1, 13, 64, 96]), top=rng.randrange(0, 33) if op == "logprobs" else 0,
                       mask=mask, scale=rng.choice([1.0, round(rng.uniform(0.5, 2.0), 3)]), ids=ids,
                       entropy=op == "logprobs_grad" and rng.random() < 0.5)
    else:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 8192 * 32000 * 1024 if dtype == "bf16" else 2048 * 16384 * 512
        while True:
            n, classes, dim = _between(rng, 1, 8192), _between(rng, 1000, 100000), _between(rng, 25, 4096)
            if rng.random() < 0.5:
                dim = max(32, dim // 32 * 32) + (32 if dim // 32 == 96 else 0)
            if n * classes * dim <= most and classes * dim <= 100000 * 2048:
                break
        case = _score("", op, dtype, n, classes, dim, scale=rng.choice([1.0, 1.0, round(rng.uniform(0.5, 1.5), 3)]), ids=ids)
    del case["name"]
    return case


# How often a class comes: class v of a table of V with probability ((v + 1) / V)^(1/4) - (v / V)^(1/4), so that a few are in
# every batch many times and most in none, as words of a text are; then the classes change places, for neighbours in
# frequency are not neighbours in a table.

def _places(classes):
    step = 7919
    while math.gcd(step, classes) != 1:
        step += 2
    return step


def _classes(case, n, gen):
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    v = (u ** 4 * case["classes"]).long().clamp_(max=case["classes"] - 1)
    return v * _places(case["classes"]) % case["classes"]


def _distinct(n, classes):
    """Different classes among n, on average."""
    v = torch.arange(classes + 1, dtype=torch.float64)
    p = torch.diff((v / classes) ** 0.25)
    return float((1.0 - torch.exp(n * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, n, classes = DTYPES[case["dtype"]], case["n"], case["classes"]
    normal = lambda *shape, std=1.0: (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)  # noqa: E731
    s = dict(case)
    ids = _classes(case, n, gen)
    if case["op"] not in ("lookup", "lookup_grad"):
        # one row in sixteen is padding, or belongs to what the model was asked and not to what it says
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 1 / 16, IGNORED, ids)
    s["ids"] = ids.to(IDS[case["ids"]])
    if case["op"] == "lookup":
        s["table"] = normal(classes, case["dim"], std=0.02)
    elif case["op"] == "lookup_grad":
        s["grad"] = normal(n, case["dim"], std=0.01)
    elif case["op"] in ("logprobs", "logprobs_grad"):
        rows = normal(n, classes + case["pad"], std=3.0)
        s["logits"] = rows[:, :classes]
        # bit v % 32 of word v / 32: class v is allowed; three quarters of the classes are
        words = lambda: torch.randint(-2**31, 2**31, (n, (classes + 31) // 32), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)  # noqa: E731
        s["allowed"] = None
        if case["mask"]:
            s["allowed"] = words() | words()
            at = ids.clamp(min=0)  # what was said was allowed
            bit = torch.ones(n, dtype=torch.int32, device="cuda") << (at & 31).to(torch.int32)
            rows = torch.arange(n, device="cuda")
            s["allowed"][rows, at >> 5] |= bit
    else:
        s["x"] = normal(n, case["dim"])
        s["weight"] = normal(classes, case["dim"], std=2.0 / math.sqrt(case["dim"]))
    if case["op"] in ("logprobs_grad", "score_grad"):
        # minus the mean log-probability, rows weighted by how well they went
        w = torch.rand(n, generator=gen, device="cuda") + 0.5
        s["grad_logprob"] = -w / n
        s["grad_entropy"] = torch.full((n,), -0.01 / n, device="cuda") if case.get("entropy") else None
    return s


def _run_own(s):
    import paper_1910_11141_amd as nuts

    op = s["op"]
    if op == "lookup":
        return nuts.nuts_lookup(s["table"], s["ids"], scale=s["scale"])
    if op == "lookup_grad":
        return nuts.nuts_lookup_grad(s["grad"], s["ids"], s["classes"], scale=s["scale"])
    if op in ("logprobs", "logprobs_grad"):
        out = nuts.nuts_logprobs(s["logits"], s["ids"], scale=s["scale"], allowed=s["allowed"], n_top=s["top"])
        if op == "logprobs":
            got = {"logprob": out.logprob, "lse": out.lse, "entropy": out.entropy}
            return {**got, "top_ids": out.top_ids, "top_logprobs": out.top_logprobs} if s["top"] else got
        grad = nuts.nuts_logprobs_grad(s["logits"], s["ids"], out.lse, out.entropy, grad_logprob=s["grad_logprob"],
                                       grad_entropy=s["grad_entropy"], scale=s["scale"], allowed=s["allowed"])
        return {"logprob": out.logprob, "entropy": out.entropy, "grad": grad}
    if op == "score":
        out = nuts.nuts_score(s["x"], s["weight"], s["ids"], scale=s["scale"])
        return {"logprob": out.logprob, "lse": out.lse, "entropy": out.entropy}
    out = nuts.nuts_score(s["x"], s["weight"], s["ids"], scale=s["scale"], keep_logits=True)
    grad_x, grad_weight = nuts.nuts_score_grad(s["x"], s["weight"], s["ids"], out.lse, out.entropy, grad_logprob=s["grad_logprob"],
                                               scale=s["scale"], logits=out.logits)
    return {"logprob": out.logprob, "grad_x": grad_x, "grad_weight": grad_weight}


def _statistics(z, ids):
    """log-probability of each row's target (0 where it has none), log of the sum, entropy; and the probabilities."""
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    p = e / total
    entropy = lse[:, 0] - (p * torch.where(p > 0, z, 0.0)).sum(dim=1)
    known = (ids >= 0) & (ids < z.shape[1])
    at = torch.where(known, ids, 0).long()
    logprob = torch.where(known, z.gather(1, at[:, None])[:, 0] - lse[:, 0], 0.0)
    return logprob, lse[:, 0], entropy, p, known, at


def _grad_logits(s, z, lse, entropy, p, known, at):
    """d/dz of sum(grad_logprob * logprob) + sum(grad_entropy * entropy)."""
    g = torch.where(known, s["grad_logprob"], 0.0)
    grad = -g[:, None] * p
    if s.get("grad_entropy") is not None:
        grad -= s["grad_entropy"][:, None] * p * torch.where(p > 0, z - lse[:, None] + entropy[:, None], 0.0)
    return grad.scatter_add_(1, at[:, None], g[:, None])


def run(s):
    if own:
        return _run_own(s)
    op, ids, scale = s["op"], s["ids"], s["scale"]
    if op == "lookup":
        return (s["table"][ids.long()].float() * scale).to(s["table"].dtype)
    if op == "lookup_grad":
        grad = s["grad"]
        table = torch.zeros(s["classes"], grad.shape[1], device=grad.device)
        return table.index_add_(0, ids.long(), grad.float()).mul_(scale).to(grad.dtype)
    if op in ("logprobs", "logprobs_grad"):
        ranked = z = s["logits"].float()
        if s["allowed"] is not None:
            v = torch.arange(s["classes"], device=z.device)
            ruled_out = (s["allowed"][:, v >> 5] >> (v & 31)) & 1 == 0
            ranked = z = z.masked_fill(ruled_out, -math.inf)
        z = z * scale
        logprob, lse, entropy, p, known, at = _statistics(z, ids)
        if op == "logprobs_grad":
            grad = _grad_logits(s, z, lse, entropy, p, known, at) * scale
            if s["allowed"] is not None:
                grad = grad.masked_fill(ruled_out, 0.0)
            return {"logprob": logprob, "entropy": entropy, "grad": grad.to(s["logits"].dtype)}
        got = {"logprob": logprob, "lse": lse, "entropy": entropy}
        if s["top"]:
            # the order of the numbers, and of their places where they are equal, as whole numbers
            bits = (ranked + 0.0).view(torch.int32)
            order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
            key = (order << 32) + (s["classes"] - torch.arange(s["classes"], device=z.device))
            top_ids = key.topk(s["top"], dim=1).indices
            got |= {"top_ids": top_ids.int(), "top_logprobs": z.gather(1, top_ids) - lse[:, None]}
        return got
    x, weight = s["x"].float(), s["weight"].float()
    z = (x @ weight.t()) * scale
    logprob, lse, entropy, p, known, at = _statistics(z, ids)
    if op == "score":
        return {"logprob": logprob, "lse": lse, "entropy": entropy}
    grad = _grad_logits(s, z, lse, entropy, p, known, at) * scale
    return {"logprob": logprob, "grad_x": (grad @ weight).to(s["x"].dtype), "grad_weight": (grad.t() @ x).to(s["x"].dtype)}


def exact(case, seed):
    """What `run` returns, in 64 bits: sums of a class's rows by a sorted order, logarithms of the softmax by torch's own."""
    s = prepare(case, seed)
    op, ids, scale = s["op"], s["ids"].long(), s["scale"]
    if op == "lookup":
        return torch.index_select(s["table"], 0, ids).double() * scale
    if op == "lookup_grad":
        # several sums of few columns: a 64-bit copy of everything at once is not needed
        order = torch.argsort(ids, stable=True)
        count = torch.bincount(ids, minlength=s["classes"])
        ends = torch.cumsum(count, 0)
        out = torch.empty(s["classes"], s["dim"], dtype=torch.float64, device="cuda")
        for c in range(0, s["dim"], 256):
            run_sum = torch.cumsum(s["grad"][order, c:c + 256].double(), 0)
            run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
            out[:, c:c + 256] = (run_sum[ends] - run_sum[ends - count]) * scale
        return out
    if op in ("logprobs", "logprobs_grad"):
        z = s["logits"].double() * scale
        if s["allowed"] is not None:
            shifts = torch.arange(32, device="cuda", dtype=torch.int32)
            bits = (s["allowed"][:, :, None] >> shifts) & 1
            z = torch.where(bits.reshape(s["n"], -1)[:, :s["classes"]] == 1, z, -math.inf)
    else:
        x, weight = s["x"].double(), s["weight"].double()
        z = (x @ weight.t()) * scale
    logp = torch.log_softmax(z, dim=1)
    lse = torch.logsumexp(z, dim=1)
    p = torch.exp(logp)
    entropy = torch.special.entr(p).sum(dim=1)
    has = (ids >= 0).double()
    at = ids.clamp(min=0)[:, None]
    logprob = torch.where(ids >= 0, logp.gather(1, at)[:, 0], 0.0)
    if op in ("logprobs", "score"):
        got = {"logprob": logprob, "lse": lse, "entropy": entropy}
        if s.get("top"):
            got |= {"top_ids": None, "top_logprobs": logp.topk(s["top"], dim=1).values}
        return got
    g = s["grad_logprob"].double() * has
    grad = p * -g[:, None]
    grad.scatter_add_(1, at, g[:, None])
    if s.get("grad_entropy") is not None:
        grad += s["grad_entropy"].double()[:, None] * (torch.special.entr(p) - p * entropy[:, None])
    grad *= scale
    if op == "logprobs_grad":
        return {"logprob": logprob, "entropy": entropy, "grad": grad}
    return {"logprob": logprob, "grad_x": grad @ weight, "grad_weight": grad.t() @ x}


def work(case):
    n, classes, size = case["n"], case["classes"], SIZES[case["dtype"]]
    id_bytes = n * (4 if case["ids"] == "i32" else 8)
    if case["op"] == "lookup":
        rows = _distinct(n, classes)
        return {"bytes": (rows + n) * case["dim"] * size + id_bytes, "flops": n * case["dim"]}
    if case["op"] == "lookup_grad":
        return {"bytes": (n + classes) * case["dim"] * size + id_bytes, "flops": n * case["dim"]}
    if case["op"] in ("logprobs", "logprobs_grad"):
        # an exponential, two sums and a maximum for each logit; the gradient has the exponential again and its product
        grad = case["op"] == "logprobs_grad"
        mask = n * ((classes + 31) // 32) * 4 if case["mask"] else 0
        rows = n * 4 * (3 + 2 * case["top"] + (1 if grad else 0))
        return {"bytes": n * classes * size * (2 if grad else 1) + mask + rows + id_bytes, "flops": n * classes * (9 if grad else 5)}
    dim, products = case["dim"], 3 if case["op"] == "score_grad" else 1
    both = (n + classes) * dim * size
    return {"bytes": both * (2 if products == 3 else 1) + 12 * n + id_bytes, "flops": 2.0 * products * n * classes * dim}
