"""What the word model does with steps and penalties, and a run of all operators together, against 64 bits."""
import math

import pytest
import torch

import categorical_ref as R
import learning_ref as L
import paper_1910_11141_amd as nuts
from test_gpu_word_model import exact, model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,max_norm", [(32, None), (32, 1.0), (8, 2.0)])
def test_steps_of_a_fit_are_adamws(bits, max_norm):
    """Each step from where the last ended: gradients in 64 bits, whose errors in 32 are 1e-5 of their norm (as in the model's own test); eps is what a step
    divides by at least, so that a parameter is off by lr / eps of that at most and by nothing else that counts."""
    m, t, w, g = model(700, 101, 7)
    before = (t.clone(), w.clone())
    moments = [(torch.zeros_like(x).double(), torch.zeros_like(x).double()) for x in (t, w)]
    steps = m.fit(3, lr=0.01, start=(t, w), max_norm=max_norm, bits=bits)
    for step, (t, w, logp) in enumerate(steps, 1):
        want_logp, *grads = exact(m, *before)
        assert abs(float(logp) - float(want_logp)) <= 1e-5 * abs(float(want_logp))
        norm = math.sqrt(sum(float(x.square().sum()) for x in grads))
        factor = min(1.0, max_norm / norm) if max_norm is not None else 1.0
        for i, (x, old, grad) in enumerate(zip((t, w), before, grads)):
            new, _, m1, _, v1, _ = L.adamw(old, grad, *moments[i], step=step, lr=0.01, weight_decay=0.0, scale=-1.0, factor=factor)
            if bits == 32:
                moments[i] = m1, v1
                # a step's length is lr, whatever the gradient's; where the gradient is off by more than a hundredth of itself it may be any
                clear = grad.abs() > 100 * 2e-5 * grad.abs().mean()
                assert float((x.double() - new)[clear].abs().max()) <= 0.01 * 0.04
            assert float((x - old).abs().max()) <= 0.01 * 8   # (moments of 8 bits are rounded at random, but a step is no longer than a few lr)
        before = (t.clone(), w.clone())
    assert step == 3


def test_answers_with_penalties():
    m, t, w, g = model()
    asked = torch.tensor([0, 5, 210], device="cuda")
    history = torch.randint(0, 211, (3, 30), generator=g, device="cuda")
    kw = dict(repetition=1.5, frequency=0.5, presence=0.25)
    ids, logprobs, entropy = m.answers(t, w, asked, n_top=4, temperature=0.8, history=history, **kw)
    logits = t[asked].double() @ w.double().t()
    seen, said = L.counts(history, None, None, 3, 211)
    z = torch.where(seen > 0, torch.where(logits > 0, logits / 1.5, logits * 1.5), logits)
    z = (z - torch.where(said > 0, 0.5 * said + 0.25, 0.0)) / 0.8
    want = torch.log_softmax(z, 1).topk(4, 1)
    assert torch.equal(ids.long(), want.indices) and float((logprobs.double() - want.values).abs().max()) < 1e-4
    plain = m.answers(t, w, asked, n_top=4)
    again = m.answers(t, w, asked, n_top=4, history=history)
    assert all(torch.equal(a, b) for a, b in zip(plain, again))


def test_texts_that_may_not_repeat_a_word():
    m, t, w, g = model(900, 40, 6)
    text = torch.tensor([[1, 2], [7, 7], [39, 0]], device="cuda")
    allowed = torch.ones(40, dtype=torch.bool, device="cuda")
    allowed[5] = False
    got = m.continue_text(t, w, text, 36, g, presence=1e6, allowed=R.pack_bits(allowed))
    assert got.shape == (3, 38) and torch.equal(got[:, :2], text)
    for row in got[:, 2:].tolist():   # 39 words may come, and none twice
        assert len(set(row)) == 36 and 5 not in row and min(row) >= 0
    assert m.continue_text(t, w, text, 0, g).equal(text)
    # with no penalties and hardly any chance: the most probable word each time
    got = m.continue_text(t, w, text, 5, g, temperature=1e-4)
    for at in range(2, 7):
        assert torch.equal(got[:, at], m.answers(t, w, got[:, at - 1], n_top=1)[0][:, 0].long())


@pytest.mark.parametrize("bits", [32, 8])
def test_all_operators_together(bits):
    """A table of logits by word with a bias of each class, trained through penalties: lookup, penalties, log-probabilities, all their gradients, the norm and a step.
    Gradients are off by some 1e-6 of 1 / n; eps = 0.01 is what a step divides by at least."""
    n, words, g = 600, 90, torch.Generator(device="cuda").manual_seed(5)
    table = torch.randn(words, words, generator=g, device="cuda")
    bias = torch.randn(words, generator=g, device="cuda")
    ids, targets = (torch.randint(0, words, (n,), generator=g, device="cuda") for _ in range(2))
    history = torch.randint(-1, words, (n, 12), generator=g, device="cuda")
    lengths = torch.randint(0, 13, (n,), generator=g, device="cuda").int()
    kw = dict(lengths=lengths, repetition=1.3)
    seen = L.counts(history, lengths, None, n, words)[0]
    said = seen.double()
    params = [table, bias]
    moments = nuts.Moments(params, bits=bits)
    state = [(torch.zeros_like(p, dtype=torch.float64), torch.zeros_like(p, dtype=torch.float64)) for p in params]
    ones = torch.full((n,), 1.0 / n, device="cuda")
    for step in range(1, 4):
        exact_p = [p.double().clone().requires_grad_() for p in params]
        x = exact_p[0][ids]
        z = torch.where(seen > 0, torch.where(x > 0, x / 1.3, x * 1.3), x) - 0.5 * said - 0.25 * (said > 0) + exact_p[1]
        loss = torch.log_softmax(z, 1).gather(1, targets[:, None]).mean()
        grads = torch.autograd.grad(loss, exact_p)

        logits = nuts.nuts_lookup(table, ids)
        adjusted = nuts.nuts_penalties(logits, history, frequency=0.5, presence=0.25, bias=bias, **kw)
        out = nuts.nuts_logprobs(adjusted, targets)
        assert abs(float(out.logprob.double().mean()) - float(loss.detach())) < 1e-5
        dz = nuts.nuts_logprobs_grad(adjusted, targets, out.lse, grad_logprob=ones)
        dx, dbias = nuts.nuts_penalties_grad(dz, logits, history, out=dz, want_bias=True, **kw)
        dtable = nuts.nuts_lookup_grad(dx, ids, words)
        for got, want in zip((dtable, dbias), grads):
            assert float((got.double() - want).norm()) <= 1e-5 * float(want.norm())
        norm = nuts.nuts_norm([dtable, dbias], max_norm=0.01)
        want_norm = math.sqrt(sum(float(x.square().sum()) for x in grads))
        assert abs(float(norm.norm) - want_norm) < 1e-5 * want_norm
        old = [p.clone() for p in params]
        nuts.nuts_adamw(moments, [dtable, dbias], step=step, lr=0.1, eps=0.01, weight_decay=0.1, scale=-1.0, factor=norm.factor, seed=7)
        for i, (p, q, grad) in enumerate(zip(params, old, grads)):
            new, _, m1, _, v1, _ = L.adamw(q.view(-1), grad.view(-1), *(s.view(-1) for s in state[i]), step=step, lr=0.1, eps=0.01, weight_decay=0.1, scale=-1.0,
                                           factor=min(1.0, 0.01 / want_norm))
            # gradients of at most 0.01 that are 1e-5 off, divided by 0.01 and times 0.1; 24 bits of numbers below 8
            assert float((p.view(-1).double() - new).abs().max()) <= 2e-6 + 4 * 8 * 2.0 ** -24
            if bits == 32:
                state[i] = m1.view(p.shape), v1.view(p.shape)
            else:   # (what the next step goes on from is what the codes stand for)
                mv = nuts.nuts_adamw_values(moments)
                state[i] = mv[0][i].double(), mv[1][i].double()
