"""Entries of the gradients that are 0 whatever the rest of their row is: classes that may not come, and classes of probability 0."""
import math

import pytest
import torch

import categorical_ref as R

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ops():
    import paper_1910_11141_amd as nuts
    return nuts


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("classes", [5, 1000, 20011])
@pytest.mark.parametrize("entropy", [False, True])
def test_classes_that_may_not_come_have_no_gradient(dtype, classes, entropy):
    nuts, g = ops(), gen(classes)
    logits = torch.randn(9, classes, generator=g, device="cuda").to(dtype)
    targets = torch.randint(0, classes, (9,), generator=g, device="cuda")
    allowed = torch.rand(9, classes, generator=g, device="cuda") < 0.5
    allowed[:, 0], allowed[:, 1] = True, False
    logits[0, 0] = math.nan                                       # the whole row has no lse
    logits[1, 0] = math.inf
    logits[2, 0], logits[2, 1] = math.nan, math.inf
    targets[2] = 1                                                # a target that may not come
    grads = [torch.randn(9, generator=g, device="cuda") for _ in range(3)]
    for part, at, value in ((0, 3, math.inf), (0, 4, math.nan), (1, 5, -math.inf), (1, 6, math.nan), (2, 7, math.inf)):
        grads[part][at] = value
    fwd = nuts.nuts_logprobs(logits, targets, allowed=R.pack_bits(allowed))
    got = nuts.nuts_logprobs_grad(logits, targets, fwd.lse, fwd.entropy, grad_logprob=grads[0], grad_lse=grads[1],
                                  grad_entropy=grads[2] if entropy else None, allowed=R.pack_bits(allowed))
    assert not bool(got[~allowed].any())
    assert bool(torch.isnan(got[:3][allowed[:3]]).all()) and bool(torch.isfinite(got[8]).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("classes", [5, 1000, 20011])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_logprobs_grad_is_0_where_the_probability_is(dtype, classes, masked, value):
    """... and in rows where every z is -infinity, also where what comes in is not finite."""
    nuts, g = ops(), gen(classes)
    logits = torch.randn(8, classes, generator=g, device="cuda").to(dtype)
    never = torch.arange(classes, device="cuda") % 2 == 1
    logits[:6, never] = -1e4
    logits[2, never] = -math.inf
    logits[6] = -math.inf                                         # empty rows
    allowed = torch.rand(8, classes, generator=g, device="cuda") < 0.7
    allowed[:, 0], allowed[7] = True, False
    if not masked:
        logits[7] = -math.inf
    targets = torch.zeros(8, dtype=torch.int64, device="cuda")
    packed = R.pack_bits(allowed) if masked else None
    fwd = nuts.nuts_logprobs(logits, targets, allowed=packed)
    for part in range(3):
        grads = [torch.randn(8, generator=g, device="cuda") for _ in range(3)]
        grads[part][1:] = value
        got = nuts.nuts_logprobs_grad(logits, targets, fwd.lse, fwd.entropy, grad_logprob=grads[0], grad_lse=grads[1], grad_entropy=grads[2],
                                      allowed=packed)
        assert not bool(got[:6, never].any()) and not bool(got[6:].any())
        assert bool(torch.isfinite(got[0]).all()) and not bool(torch.isfinite(got[1:6, 0]).any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,classes,dim", [(3, 1000, 9), (300, 700, 40), (600, 3000, 130)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("kept", [True, False])
def test_score_grad_of_classes_of_probability_0(dtype, n, classes, dim, value, kept):
    """Weights of classes that no row can have get no gradient, and one row's gradient that is not finite reaches no other row."""
    nuts, g = ops(), gen(n)
    x, w = (torch.randn(rows, dim, generator=g, device="cuda").to(dtype) for rows in (n, classes))
    never = torch.arange(classes, device="cuda") % 2 == 1
    x[:, 0], w[:, 0] = 1.0, torch.where(never, -8192.0, 0.0).to(dtype)
    targets = torch.randint(0, classes // 2, (n,), generator=g, device="cuda") * 2
    fwd = nuts.nuts_score(x, w, targets, keep_logits=True)
    for part in range(3):
        grads = [torch.randn(n, generator=g, device="cuda") for _ in range(3)]
        call = lambda: nuts.nuts_score_grad(x, w, targets, fwd.lse, fwd.entropy, grad_logprob=grads[0], grad_lse=grads[1], grad_entropy=grads[2],
                                            logits=fwd.logits if kept else None)
        clean_x, _ = call()
        grads[part][1] = value
        got_x, got_w = call()
        others = torch.arange(n, device="cuda") != 1
        assert not bool(got_w[never].any()) and not bool(torch.isfinite(got_w[~never]).all())
        assert torch.equal(got_x[others], clean_x[others]) and not bool(torch.isfinite(got_x[1]).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("classes", [5, 1000, 20011])
@pytest.mark.parametrize("lse", [3.0, -500.0, 5000.0])
def test_a_part_of_the_classes_of_which_none_may_come_has_no_gradient(dtype, classes, lse):
    """With the lse of a longer row, which is finite, and near 0 or far from it."""
    nuts, g = ops(), gen(classes)
    logits = torch.randn(3, classes, generator=g, device="cuda").to(dtype)
    logits[1] = -math.inf
    allowed = torch.ones(3, classes, dtype=torch.bool, device="cuda")
    allowed[0] = False
    allowed[2] = False
    logits[2] = -math.inf
    ones = torch.ones(3, device="cuda")
    for mask in (None, R.pack_bits(allowed)):
        got = nuts.nuts_logprobs_grad(logits, torch.full((3,), -1, device="cuda"), ones * lse, ones * 2.0, grad_lse=ones, grad_entropy=ones, allowed=mask)
        assert not bool(got[1:].any()) and (mask is None or not bool(got[0].any()))
