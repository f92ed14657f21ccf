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
