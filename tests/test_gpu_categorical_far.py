"""Gradients of rows whose logits lie far from 0, where the logarithm of their sum has few digits left for the sum itself.

The logits of these tests are exact, so bounds do not grow with them: log p = s (x - m) - ln S has the roundings of the
difference, of its product and of the sum (5 u |log p| with that by log2 e), ln S the error TOL of tests/test_gpu_categorical.py, and
lse, where it is used in place of both, half a unit in its last place (2^-19 up to 64 for binary32, 2^-15 up to 1024 for 16 bits): in
all less than 2 TOL + 6 u |log p|, relative to p.  The entropy is off by 30 TOL."""
import math

import pytest
import torch

import categorical_ref as R

pytestmark = pytest.mark.gpu

TOL = 4e-5
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ops():
    import paper_1910_11141_amd as nuts
    return nuts


def _bound(want, z, targets, scale, parts, dtype):
    """What the gradient `want` with respect to exact logits may be off by, rounded to `dtype`."""
    _, _, entropy, p = R.logprobs(z, targets)
    log_p = torch.where(p == 0, torch.zeros_like(p), torch.log(p.clamp(min=1e-300))).abs()
    rel = 2 * TOL + 6 * R.U * log_p
    total = (parts[0].double().abs() + parts[1].double().abs())[:, None]
    h = parts[2].double().abs()[:, None] * (log_p + entropy[:, None] + 60)
    bound = (p * (total + h) * rel + R.U * 4 * total * (p > 0)) * scale + want.abs() * 4 * R.U
    return bound + (want.abs() + bound) * R.EPS[dtype] * 1.01 + R.TINY[dtype] + 2.0 ** -126


FAR = [0.0, 40.0, 100.0, -300.0, 1e3, 6e4, -6e4, 1e6, 1e8, -1e9, 2.0 ** 27, 3e30, -3e38]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,classes", [(3, 4), (2, 1000), (5, 5000), (3, 20011), (300, 700)])
@pytest.mark.parametrize("masked", [False, True])
def test_logprobs_grad_of_rows_far_from_0(dtype, n, classes, masked):
    nuts, g = ops(), gen(n + classes)
    for shift in FAR:
        if dtype == torch.float16 and abs(shift) > 6e4:
            continue
        for scale in (1.0, 0.8):
            logits = (torch.randn(n, classes, generator=g, device="cuda", dtype=torch.float64) * 3 + shift).to(dtype)
            targets = torch.randint(-1, classes, (n,), generator=g, device="cuda")
            allowed = None
            if masked:
                allowed = torch.rand(n, classes, generator=g, device="cuda") < 0.6
                allowed[:, 0] = True
            packed = None if allowed is None else R.pack_bits(allowed)
            parts = [torch.randn(n, generator=g, device="cuda") for _ in range(3)]
            fwd = nuts.nuts_logprobs(logits, targets, scale=scale, allowed=packed)
            got = nuts.nuts_logprobs_grad(logits, targets, fwd.lse, fwd.entropy, grad_logprob=parts[0], grad_lse=parts[1],
                                          grad_entropy=parts[2], scale=scale, allowed=packed)
            s = torch.tensor(scale, dtype=torch.float32).double().item()
            z = logits.double() * s
            if allowed is not None:
                z = torch.where(allowed, z, torch.full_like(z, -math.inf))
            want = R.grad_logits(z, targets, allowed, s, *parts)
            off = (got.double() - want).abs() - _bound(want, z, targets, s, parts, dtype)
            assert float(off.max()) <= 0, (shift, scale, float(off.max()))


@pytest.mark.parametrize("classes", [4, 1000, 30000])
@pytest.mark.parametrize("far", [1e5, -1e6, 1e7, 2.0 ** 27, -1e9])
def test_probabilities_of_far_rows_add_up_to_1(classes, far):
    nuts = ops()
    logits = torch.full((2, classes), far, device="cuda")
    logits[1] += torch.randn(classes, generator=gen(1), device="cuda") * 3
    targets = torch.tensor([0, classes - 1], device="cuda")
    fwd = nuts.nuts_logprobs(logits, targets)
    grad = nuts.nuts_logprobs_grad(logits, targets, fwd.lse, grad_logprob=torch.ones(2, device="cuda")).double()
    assert float((grad[0, 1:] * classes + 1).abs().max()) <= 2 * TOL
    # p's sum is 1 but for the same relative error of each, and each entry's rounding (the target's: of numbers up to 1)
    assert float(grad.sum(1).abs().max()) <= 2 * TOL + 4 * R.U


def test_binary32_gradients_of_short_rows_lose_nothing_to_lse():
    """Rows that a workgroup holds: half a unit in lse's last place, here 32 u, does not reach p = 2^w / S.  The 2-norm is that of the
    largest p, with |x - m| below 6: two roundings of w (6 u each), 2 u of the exponential and of the quotient, and of S's sum,
    whose terms' errors of either sign add up to less than one of them, as much as of one term: 8 u where they are as often up as down."""
    nuts, g = ops(), gen(3)
    logits = torch.randn(500, 1000, generator=g, device="cuda") * 3 + 40
    targets = torch.randint(0, 1000, (500,), generator=g, device="cuda")
    weight = torch.rand(500, generator=g, device="cuda") + 0.5
    fwd = nuts.nuts_logprobs(logits, targets)
    assert bool(((fwd.lse > 32) & (fwd.lse < 64)).all())
    grad = nuts.nuts_logprobs_grad(logits, targets, fwd.lse, grad_logprob=weight)
    want = R.grad_logits(logits.double(), targets, None, 1.0, weight)
    others = torch.ones_like(want, dtype=torch.bool).scatter_(1, targets[:, None], False)  # (the target's is g - g p)
    assert float((grad.double() - want)[others].norm()) <= 8 * R.U * float(want[others].norm())


def _far_scores(n, classes, dim, shift, dtype, seed):
    """Features and weights of small whole numbers, and one that takes all scores `shift` away from 0; every score and every part of its sum
    is a multiple of four units in its last place, so that binary32 products are exact."""
    g = gen(seed)
    unit = max(0.25, 2.0 ** (math.floor(math.log2(abs(shift))) - 23 + 2)) if shift else 0.25
    x = torch.randint(-2, 3, (n, dim), generator=g, device="cuda").to(dtype)
    w = torch.randint(-2, 3, (classes, dim), generator=g, device="cuda").to(dtype) * unit
    x[:, 0], w[:, 0] = 1.0, shift
    targets = torch.randint(-1, classes, (n,), generator=g, device="cuda")
    return x, w, targets, [torch.randn(n, generator=g, device="cuda") for _ in range(3)]


def _check_far_rows(x, w, targets, parts, rows, grad_x, dtype):
    """The gradient with respect to some rows of x against 64 bits; returns what they add to the weights' and what that may be off by."""
    z = x[rows].double() @ w.double().t()
    own = [p[rows] for p in parts]
    dz = R.grad_logits(z, targets[rows], None, 1.0, *own)
    dz_off = _bound(dz, z, targets[rows], 1.0, own, dtype)
    want_x = dz @ w.double()
    bound_x = dz_off @ w.double().abs() + (dz.abs() @ w.double().abs()) * (w.shape[0] + 2) * R.U
    bound_x = bound_x * 1.01 + (want_x.abs() + bound_x) * R.EPS[dtype] * 1.01
    off = ((grad_x[rows].double() - want_x).abs() - bound_x).amax(0)
    assert float(off.max()) <= 0, off
    bound_w = dz_off.t() @ x[rows].double().abs() + (dz.abs().t() @ x[rows].double().abs()) * (x.shape[0] + 2) * R.U
    return dz.t() @ x[rows].double(), bound_w


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,classes,dim", [(3, 1000, 9), (300, 5000, 40), (2, 20011, 16), (600, 3000, 130)])
@pytest.mark.parametrize("shift", [0.0, 128.0, -2.0 ** 13, 2.0 ** 20, -2.0 ** 27])
@pytest.mark.parametrize("kept", [True, False])
def test_score_grad_of_rows_far_from_0(dtype, n, classes, dim, shift, kept):
    nuts = ops()
    x, w, targets, parts = _far_scores(n, classes, dim, shift, dtype, n + dim)
    fwd = nuts.nuts_score(x, w, targets, keep_logits=True)
    assert torch.equal(fwd.logits.double(), x.double() @ w.double().t())
    grad_x, grad_w = nuts.nuts_score_grad(x, w, targets, fwd.lse, fwd.entropy, grad_logprob=parts[0], grad_lse=parts[1], grad_entropy=parts[2],
                                          logits=fwd.logits if kept else None)
    want_w, bound_w = _check_far_rows(x, w, targets, parts, slice(0, n), grad_x, dtype)
    bound_w = bound_w * 1.01 + (want_w.abs() + bound_w) * R.EPS[dtype] * 1.01
    assert float(((grad_w.double() - want_w).abs() - bound_w).max()) <= 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kept", [True, False])
def test_score_grad_of_some_far_rows_over_several_pieces(dtype, kept):
    """More scores than one piece of the classes holds: rows that begin far from 0, and one that does alone among its neighbours."""
    nuts = ops()
    n, classes, dim = 65536 + 40, 9000, 32
    x, w, targets, parts = _far_scores(n, classes, dim, 2.0 ** 20, dtype, 5)
    far = torch.zeros(n, dtype=torch.bool, device="cuda")
    far[:700], far[30000], far[n - 1] = True, True, True
    w[:, 1:] = w[:, 1:].sign() * 0.25
    x[~far, 0] = 0.0
    fwd = nuts.nuts_score(x, w, targets, keep_logits=kept)
    grad_x, grad_w = nuts.nuts_score_grad(x, w, targets, fwd.lse, fwd.entropy, grad_logprob=parts[0], grad_lse=parts[1], grad_entropy=parts[2],
                                          logits=fwd.logits)
    want_w, bound_w = 0.0, 0.0
    for r in range(0, n, 8192):
        rows = slice(r, min(r + 8192, n))
        some_w, some_bound = _check_far_rows(x, w, targets, parts, rows, grad_x, dtype)
        want_w, bound_w = want_w + some_w, bound_w + some_bound
    bound_w = bound_w * 1.01 + (want_w.abs() + bound_w) * R.EPS[dtype] * 1.01
    assert float(((grad_w.double() - want_w).abs() - bound_w).max()) <= 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("classes", [1000, 4000, 20000])
@pytest.mark.parametrize("shift", [0.0, -100.0, 1000.0])
def test_logprobs_grad_of_a_part_of_the_classes(dtype, classes, shift):
    """A row's classes in two parts, each with the whole row's lse and entropy: the parts of its gradient.  lse's rounding is an error of p here
    however it is used: half a unit in the last place of 1000 and some is 2^-14 at most, with which the bound's 2 TOL = 2^-13.6 still holds the rest."""
    nuts, g = ops(), gen(classes)
    logits = (torch.randn(6, classes, generator=g, device="cuda") * 3 + shift).to(dtype)
    targets = torch.randint(0, classes, (6,), generator=g, device="cuda")
    parts = [torch.randn(6, generator=g, device="cuda") for _ in range(3)]
    fwd = nuts.nuts_logprobs(logits, targets)
    cut = classes * 2 // 5
    got = [nuts.nuts_logprobs_grad(logits[:, own], targets - own.start, fwd.lse, fwd.entropy, grad_logprob=parts[0], grad_lse=parts[1], grad_entropy=parts[2])
           for own in (slice(0, cut), slice(cut, classes))]
    want = R.grad_logits(logits.double(), targets, None, 1.0, *parts)
    # (a target in the other part: this part's classes lose their share all the same, from grad_lse)
    known = [(targets >= 0) & (targets < cut), targets >= cut]
    lost = [torch.where(k, 0.0, parts[0]).double()[:, None] for k in known]
    p = torch.softmax(logits.double(), 1)
    want = torch.cat([want[:, :cut] + lost[0] * p[:, :cut], want[:, cut:] + lost[1] * p[:, cut:]], 1)
    off = (torch.cat(got, 1).double() - want).abs() - _bound(want, logits.double(), targets, 1.0, parts, dtype)
    assert float(off.max()) <= 0, float(off.max())
