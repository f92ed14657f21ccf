"""The categorical operators at sizes at which they take other ways: outputs past the caches, long sorts of long rows, batches in pieces.

Bounds are those of tests/test_gpu_categorical.py and tests/categorical_ref.py."""
import pytest
import torch

import categorical_ref as R
import test_gpu_categorical as T

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ops():
    import paper_1910_11141_amd as nuts
    return nuts


@pytest.mark.parametrize("dtype,n,dim", [(torch.bfloat16, 40000, 2049), (torch.float16, 70000, 1000), (torch.float32, 33000, 1025), (torch.float32, 5000000, 7)])
def test_lookup_past_the_caches(dtype, n, dim):
    """Rows of 128 MiB and more, at addresses that suit an element and no more."""
    nuts, g = ops(), gen(n)
    assert n * dim * dtype.itemsize >= 1 << 27
    table = torch.randn(3001, dim, generator=g, device="cuda").to(dtype)
    ids = torch.randint(-3, 3004, (n,), generator=g, device="cuda")
    known = (ids >= 0) & (ids < 3001)
    want = torch.where(known[:, None], (table[torch.where(known, ids, 0)].float() * 1.5), 0.0).to(dtype)
    room = torch.full((n, dim + 3), 7.0, dtype=dtype, device="cuda")
    nuts.nuts_lookup(table, ids, scale=1.5, out=room[:, 1:dim + 1])
    assert torch.equal(room[:, 1:dim + 1], want) and bool((room[:, 0] == 7).all()) and bool((room[:, dim + 1:] == 7).all())


# digits to sort by: one, two, and two with more counts than each workgroup adds up for itself
@pytest.mark.parametrize("dtype,n,classes,dim", [(torch.bfloat16, 65600, 1500, 2049), (torch.bfloat16, 65600, 70001, 2049), (torch.float32, 131100, 1500, 1030),
                                                 (torch.float32, 131100, 70001, 1030), (torch.float32, 131000, 300001, 260)])
@pytest.mark.parametrize("kind", ["skewed", "one", "outside"])
def test_lookup_grad_of_many_long_rows(dtype, n, classes, dim, kind):
    """Rows of 1 KB and more, which whole workgroups clear, in chunks of several batches and in more than one slice of columns."""
    nuts, g = ops(), gen(n + classes)
    grad = torch.randn(n, dim, generator=g, device="cuda").to(dtype)
    ids = T._ids(kind, n, classes, g)
    out = torch.full((classes, dim + 2), 3.0, dtype=dtype, device="cuda")
    nuts.nuts_lookup_grad(grad, ids, classes, scale=0.75, out=out[:, 1:dim + 1])
    assert bool((out[:, 0] == 3).all()) and bool((out[:, dim + 1] == 3).all())
    # (64 bits, on the CPU, for the classes that come; the others are 0)
    known = (ids >= 0) & (ids < classes)
    there, back = ids[known].unique(return_inverse=True)
    want, bound = R.lookup_grad(grad[known].cpu(), back.cpu(), len(there), 0.75)
    got = out[:, 1:dim + 1]
    assert bool(((got[there].cpu().double() - want).abs() <= bound).all())
    absent = torch.ones(classes, dtype=torch.bool, device="cuda")
    absent[there] = False
    assert not bool(got[absent].any())
    old = torch.randn(classes, dim, generator=g, device="cuda").to(dtype)
    into = old.clone()
    nuts.nuts_lookup_grad(grad, ids, classes, scale=0.75, out=into, accumulate=True)
    assert torch.equal(into[absent], old[absent])
    # what is added to is rounded once more: to the sum's places, and to those of the type
    there_old = old[there].cpu().double()
    bound = bound + R.U * (there_old.abs() + want.abs()) + (want + there_old).abs() * R.EPS[dtype] * 1.01
    assert bool(((into[there].cpu().double() - (want + there_old)).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_score_in_pieces_of_rows(dtype):
    """More statistics than one piece of the rows has room for: rows on both sides of where pieces may end, and the last."""
    nuts, g = ops(), gen(41)
    n, classes, dim = 1 << 20, 4100, 8
    x = torch.randn(n, dim, generator=g, device="cuda").to(dtype)
    w = torch.randn(classes, dim, generator=g, device="cuda").to(dtype)
    targets = torch.randint(-1, classes + 1, (n,), generator=g, device="cuda")
    got = nuts.nuts_score(x, w, targets, scale=0.8)
    s = torch.tensor(0.8, dtype=torch.float32).double().item()
    for first in range(0, n, 1 << 16):
        rows = slice(first, first + (1 << 16))
        z, off = T._score_bounds(x[rows], w, s)
        logprob, lse, entropy, _ = R.logprobs(z, targets[rows])
        worst = off.amax(1)
        assert bool(((got.lse[rows].double() - lse).abs() <= worst + T.TOL + 2 * R.U * lse.abs()).all())
        assert bool(((got.logprob[rows].double() - logprob).abs() <= 2 * worst + T.TOL + 2 * R.U * logprob.abs()).all())
        assert bool(((got.entropy[rows].double() - entropy).abs() <= 30 * T.TOL + 60 * worst).all())
        del z, off
    kept = nuts.nuts_score(x, w, targets, scale=0.8, keep_logits=True)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], kept[:3]))
    for first in range(0, n, 1 << 16):
        z, off = T._score_bounds(x[first:first + 4096], w, s)
        assert bool(((kept.logits[first:first + 4096].double() - z).abs() <= off).all())


@pytest.mark.parametrize("kept", [True, False])
def test_score_grad_of_bfloat16_over_several_pieces(kept):
    """What the targets' entries of dZ lose in their rounding is made up for in every piece of the classes: the gradients are as far off as
    rounding the exact ones makes them, and a tenth (as in test_score_grad_loses_nothing_to_dz_of_8_bits)."""
    nuts, g = ops(), gen(42)
    n, classes, dim = 65536 + 40, 9000, 64
    x = torch.randn(n, dim, generator=g, device="cuda").bfloat16()
    w = (torch.randn(classes, dim, generator=g, device="cuda") / 8).bfloat16()
    targets = torch.randint(0, classes, (n,), generator=g, device="cuda")
    weight = torch.randn(n, generator=g, device="cuda")
    fwd = nuts.nuts_score(x, w, targets, keep_logits=kept)
    grad_x, grad_w = nuts.nuts_score_grad(x, w, targets, fwd.lse, grad_logprob=weight, logits=fwd.logits)
    want_w = torch.zeros(classes, dim, dtype=torch.float64, device="cuda")
    off = least = 0.0
    for r in range(0, n, 8192):
        rows = slice(r, min(r + 8192, n))
        dz = R.grad_logits(x[rows].double() @ w.double().t(), targets[rows], None, 1.0, weight[rows])
        want_x = dz @ w.double()
        off += float((grad_x[rows].double() - want_x).square().sum())
        least += float((want_x.bfloat16().double() - want_x).square().sum())
        want_w += dz.t() @ x[rows].double()
    assert off <= 1.1 ** 2 * least
    for first in range(0, classes, 1000):  # (each piece by itself)
        own = slice(first, first + 1000)
        assert float((grad_w[own].double() - want_w[own]).norm()) <= 1.1 * float((want_w[own].bfloat16().double() - want_w[own]).norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,classes,dim", [(64, 70001, 1030), (3, 70001, 1030), (8200, 8300, 33), (8200, 8300, 34)])
@pytest.mark.parametrize("kept", [True, False])
def test_score_grad_past_the_caches(dtype, n, classes, dim, kept):
    """A weights' gradient, by the products or of few rows, and a dZ of 128 MiB and more."""
    T.test_score_grad(dtype, n, classes, dim, kept)


@pytest.mark.parametrize("kept", [True, False])
def test_score_grad_of_peaked_rows(kept):
    """Where another class than the target is nearly certain, its entry of dZ keeps its rounding to 8 bits.  Of dX = g (w_y - sum p w) that is
    sum p^2 / (1 + sum p^2) of the square, at most half, with the same relative error as the rounding of dX itself: sqrt(3/2) = 1.23 times
    that in all, and of dW likewise; 1.5 leaves a fifth to chance."""
    nuts, g = ops(), gen(43)
    n, classes, dim = 700, 3000, 128
    x = torch.randn(n, dim, generator=g, device="cuda").bfloat16()
    w = torch.randn(classes, dim, generator=g, device="cuda").bfloat16()
    targets = torch.randint(0, classes, (n,), generator=g, device="cuda")
    weight = torch.randn(n, generator=g, device="cuda")
    fwd = nuts.nuts_score(x, w, targets, keep_logits=kept)
    got = nuts.nuts_score_grad(x, w, targets, fwd.lse, grad_logprob=weight, logits=fwd.logits)
    z = x.double() @ w.double().t()
    assert float(torch.softmax(z, 1).amax(1).median()) > 0.8
    dz = R.grad_logits(z, targets, None, 1.0, weight)
    for a, want in zip(got, (dz @ w.double(), dz.t() @ x.double())):
        least = float((want.bfloat16().double() - want).norm())
        assert float((a.double() - want).norm()) <= 1.5 * least


def test_results_are_no_part_of_autograds_graph():
    nuts = ops()
    table = torch.randn(50, 16, device="cuda", requires_grad=True)
    ids = torch.arange(40, device="cuda")
    rows = nuts.nuts_lookup(table, ids)
    out = nuts.nuts_score(rows, table, ids, keep_logits=True)
    assert not any(t.requires_grad for t in (rows, *out, *nuts.nuts_score_grad(rows, table, ids, out.lse, grad_logprob=torch.ones(40, device="cuda"))))
