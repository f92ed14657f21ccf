"""The gradient of a shared bias over very many rows: no class is summed one row behind the other for as long as there are rows."""
import pytest
import torch

import paper_1910_11141_amd as nuts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,classes", [(4_000_000, 16), (1_500_000, 100)])
def test_sums_of_millions_of_rows(n, classes):
    """Gradients of one sign and size, whose roundings go the same way for long.  A sum is off by a rounding for each of the 128 rows that a workgroup adds up
    at most, of the 16 workgroups that a thread joins, of 64 such threads (6 steps), and of what is joined in the end, 31 sums at most, by as many (1 and 6): 157 U."""
    values = torch.linspace(0.6, 1.0, classes, device="cuda")
    grad = values.expand(n, -1).contiguous()
    _, bias = nuts.nuts_penalties_grad(grad, grad, want_logits=False, want_bias=True)
    want = values.double() * n
    assert float(((bias.double() - want).abs() / want).max()) <= 157 * 2.0 ** -24


@pytest.mark.parametrize("n", [127, 128, 129, 98304, 98305, 98304 * 2, 98304 * 2 + 1, 300_000, 786_432, 786_433])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_workgroups_just_hold(n, dtype):
    """Whole numbers, whose sums below 2^24 are exact: none is lost between two workgroups or counted twice."""
    classes, g = 37, torch.Generator(device="cuda").manual_seed(n)
    grad = torch.randint(-8, 9, (n, classes), generator=g, device="cuda").to(dtype)
    history = torch.randint(0, classes, (n, 2), generator=g, device="cuda")
    want = grad.double().sum(0)
    for kw in ({}, dict(history=history), dict(history=history[0])):
        again = [nuts.nuts_penalties_grad(grad, grad, want_bias=True, repetition=2.0, **kw)[1] for _ in range(2)]
        assert torch.equal(again[0].double(), want) and torch.equal(*again)


@pytest.mark.parametrize("n,classes", [(150_000, 4100), (131_073, 4096), (130_000, 12300)])
def test_many_groups_of_more_classes_than_a_slice(n, classes):
    """As above, joined in two launches of which each has several workgroups beside each other, by 16 and by 64 classes."""
    g = torch.Generator(device="cuda").manual_seed(n)
    grad = torch.randint(-8, 9, (n, classes), generator=g, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    want = torch.zeros(classes, dtype=torch.float64, device="cuda")
    for part in grad.split(10_000):
        want += part.double().sum(0)
    bias = nuts.nuts_penalties_grad(grad, grad, want_logits=False, want_bias=True)[1]
    assert torch.equal(bias.double(), want)
