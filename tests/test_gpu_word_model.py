"""The word model: its log density and gradient against 64 bits, its trajectories against what leapfrog steps do, its answers."""
import math

import pytest
import torch

import categorical_ref as R

pytestmark = pytest.mark.gpu


def model(n_pairs=900, n_words=211, dim=12, seed=1, **kw):
    from paper_1910_11141_amd import word_model
    g = torch.Generator(device="cuda").manual_seed(seed)
    words, next_words, t, w = word_model.synthetic_pairs(n_pairs, n_words, dim, g)
    return word_model.WordModel(words, next_words, n_words, dim, **kw), t, w, g


def exact(m, t, w):
    """log p and its gradients in 64 bits."""
    t, w = t.double(), w.double()
    x = t[m.words] * m.scale
    z = x @ w.t()
    logprob = R.logprobs(z, m.next_words)[0]
    dz = R.grad_logits(z, m.next_words, None, 1.0, torch.ones_like(logprob))
    k = 1.0 / m.prior_scale ** 2
    grad_t = torch.zeros_like(t).index_add_(0, m.words, dz @ w) * m.scale - k * t
    return logprob.sum() - 0.5 * k * (t.square().sum() + w.square().sum()), grad_t, dz.t() @ x - k * w


@pytest.mark.parametrize("n_pairs,n_words,dim", [(900, 211, 12), (1, 5, 3), (5000, 1300, 33)])
def test_log_density_and_gradient(n_pairs, n_words, dim):
    m, t, w, _ = model(n_pairs, n_words, dim, scale=0.7, prior_scale=1.5)
    for got, want in zip(m.log_density(t, w), exact(m, t, w)):
        # sums of some thousand terms of 24 bits, whose errors add up in no one direction
        assert float((got.double() - want).norm()) <= 1e-5 * float(want.norm())


def test_trajectories_are_reversible_and_their_energy_error_falls_with_the_square_of_the_step():
    m, t, w, g = model()
    state = (t, w, *m.log_density(t, w))
    momentum = tuple(torch.randn(t.shape, generator=g, device="cuda") for _ in range(2))
    start = float(m.energy(state, momentum))
    errors = []
    for halvings in range(2):
        end, r = m.leapfrog(state, momentum, 0.04 / 2 ** halvings, 8 * 2 ** halvings)
        errors.append(abs(float(m.energy(end, r)) - start))
    assert errors[1] < errors[0] / 2.5 and errors[0] < 50
    back, r = m.leapfrog(end, (-r[0], -r[1]), 0.02, 16)
    assert float((back[0] - t).abs().max()) < 1e-3 and float((back[1] - w).abs().max()) < 1e-3


def test_sampling_reaches_the_density_of_what_drew_the_pairs():
    m, t, w, g = model(4000, 150, 6)
    known = float(m.log_density(t, w)[0])
    got = list(m.sample(60, 0.03, 10, g))
    accepted = sum(s[3] for s in got)
    assert accepted >= 30
    assert got[0][2] < known and got[-1][2] > got[0][2] + 0.7 * (known - got[0][2])


def test_answers():
    m, t, w, _ = model()
    asked = torch.tensor([0, 5, 210], device="cuda")
    allowed = torch.ones(211, dtype=torch.bool, device="cuda")
    allowed[::4] = False
    ids, logprobs, entropy = m.answers(t, w, asked, n_top=4, allowed=R.pack_bits(allowed), temperature=0.8)
    z = torch.where(allowed, (t[asked].double() @ w.double().t()) / 0.8, -math.inf)
    lse = torch.logsumexp(z, 1)
    want = (z - lse[:, None]).topk(4, 1)
    assert torch.equal(ids.long(), want.indices) and float((logprobs.double() - want.values).abs().max()) < 1e-4
    p = torch.exp(z - lse[:, None])
    assert float((entropy.double() - torch.special.entr(p).sum(1)).abs().max()) < 1e-4
