"""A small Bayesian model of the next word, put together from the categorical operators and sampled with leapfrog steps.

Every word v has a row of features T[v] and a row of weights W[v]; the word after v is drawn from softmax(s T[v] W').  With
priors N(0, prior_scale^2) on all entries the log density of (T, W) given n observed pairs is

    log p = sum_i logprob_i - (|T|^2 + |W|^2) / (2 prior_scale^2),

the categorical counterpart of the sampler's logistic regression (Section 4.1 of the paper), whose gradient is that of the lookup, of the
scores and of the prior.  `sample` moves (T, W) by Hamiltonian trajectories of a fixed number of leapfrog steps, accepted or not by the
energy's change; `answers` asks a model for its most probable next words.

    python -m paper_1910_11141_amd.word_model            # draws pairs from a known model, samples, compares
"""
from __future__ import annotations

import argparse
import math

import torch

import paper_1910_11141_amd as nuts


class WordModel:
    """Pairs (word, next word) as int tensors on the GPU; parameters are binary32 [n_words, dim] matrices (T, W)."""

    def __init__(self, words, next_words, n_words, dim, *, scale=1.0, prior_scale=1.0):
        if words.shape != next_words.shape or words.dim() != 1:
            raise ValueError("words and next_words must be vectors of one length")
        self.words, self.next_words = words.contiguous(), next_words.contiguous()
        self.n_words, self.dim, self.scale, self.prior_scale = int(n_words), int(dim), float(scale), float(prior_scale)
        self._ones = torch.ones(words.shape[0], dtype=torch.float32, device=words.device)

    def draw_prior(self, generator):
        shape = (2, self.n_words, self.dim)
        t, w = torch.randn(shape, generator=generator, device=self.words.device).mul_(self.prior_scale).unbind(0)
        return t.contiguous(), w.contiguous()

    def log_density(self, t, w):
        """(log p as a binary64 scalar tensor, gradient with respect to T, gradient with respect to W)."""
        x = nuts.nuts_lookup(t, self.words, scale=self.scale)
        out = nuts.nuts_score(x, w, self.next_words, keep_logits=True)
        grad_x, grad_w = nuts.nuts_score_grad(x, w, self.next_words, out.lse, grad_logprob=self._ones, logits=out.logits)
        grad_t = nuts.nuts_lookup_grad(grad_x, self.words, self.n_words, scale=self.scale)
        precision = 1.0 / self.prior_scale ** 2
        prior = -0.5 * precision * (t.double().square().sum() + w.double().square().sum())
        return out.logprob.double().sum() + prior, grad_t.sub_(t, alpha=precision), grad_w.sub_(w, alpha=precision)

    def leapfrog(self, state, momentum, step_size, n_steps):
        """n_steps leapfrog steps from `state` = (T, W, log p, gradients); returns the new state and momentum."""
        t, w, logp, grad_t, grad_w = state
        t, w = t.clone(), w.clone()
        r_t, r_w = momentum[0].clone(), momentum[1].clone()
        for _ in range(n_steps):
            r_t.add_(grad_t, alpha=0.5 * step_size)
            r_w.add_(grad_w, alpha=0.5 * step_size)
            t.add_(r_t, alpha=step_size)
            w.add_(r_w, alpha=step_size)
            logp, grad_t, grad_w = self.log_density(t, w)
            r_t.add_(grad_t, alpha=0.5 * step_size)
            r_w.add_(grad_w, alpha=0.5 * step_size)
        return (t, w, logp, grad_t, grad_w), (r_t, r_w)

    @staticmethod
    def energy(state, momentum):
        return -state[2] + 0.5 * (momentum[0].double().square().sum() + momentum[1].double().square().sum())

    def sample(self, n_iters, step_size, n_steps, generator, start=None):
        """Yields (T, W, log p, accepted) after each of n_iters trajectories."""
        t, w = start if start is not None else self.draw_prior(generator)
        state = (t, w, *self.log_density(t, w))
        for _ in range(n_iters):
            momentum = tuple(torch.randn(t.shape, generator=generator, device=t.device) for _ in range(2))
            proposal, end = self.leapfrog(state, momentum, step_size, n_steps)
            change = float(self.energy(proposal, end) - self.energy(state, momentum))
            u = float(torch.rand((), generator=generator, device=t.device))
            accepted = math.log(max(u, 1e-300)) < -change  # (false for a change that is not a number)
            if accepted:
                state = proposal
            yield state[0], state[1], float(state[2]), accepted

    def answers(self, t, w, words, *, n_top=5, allowed=None, temperature=1.0):
        """The n_top most probable words after each of `words`, their log-probabilities, and how uncertain the model is (entropies)."""
        x = nuts.nuts_lookup(t, words, scale=self.scale)
        logits = nuts.nuts_score(x, w, keep_logits=True).logits
        out = nuts.nuts_logprobs(logits, scale=1.0 / temperature, allowed=allowed, n_top=n_top)
        return out.top_ids, out.top_logprobs, out.entropy


def synthetic_pairs(n_pairs, n_words, dim, generator, *, prior_scale=1.0):
    """Pairs drawn from a model of known (T, W): some words come far more often than others.  Returns (words, next words, T, W)."""
    t, w = (torch.randn((n_words, dim), generator=generator, device="cuda") * prior_scale for _ in range(2))
    words = (torch.rand(n_pairs, generator=generator, device="cuda") ** 3 * n_words).long().clamp_(max=n_words - 1)
    logits = nuts.nuts_score(nuts.nuts_lookup(t, words), w, keep_logits=True).logits
    # the largest of logits plus Gumbel noise is a draw from their softmax
    noise = -torch.log(-torch.log(torch.rand(logits.shape, generator=generator, device="cuda").clamp_(1e-20, 1 - 1e-7)))
    return words, nuts.nuts_logprobs(logits + noise, n_top=1).top_ids[:, 0].long(), t, w


def main(argv=None):
    ap = argparse.ArgumentParser(description="Samples a small Bayesian model of the next word.")
    ap.add_argument("--words", type=int, default=1000)
    ap.add_argument("--dim", type=int, default=8)
    ap.add_argument("--pairs", type=int, default=10000)
    ap.add_argument("--iterations", type=int, default=80)
    ap.add_argument("--step-size", type=float, default=0.006)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    words, next_words, true_t, true_w = synthetic_pairs(a.pairs, a.words, a.dim, g)
    model = WordModel(words, next_words, a.words, a.dim)
    known = float(model.log_density(true_t, true_w)[0])
    print(f"{a.pairs} pairs of {a.words} words; log density of the parameters that drew them {known:.0f}")
    accepted = 0
    for i, (t, w, logp, ok) in enumerate(model.sample(a.iterations, a.step_size, a.steps, g)):
        accepted += ok
        if (i + 1) % max(1, a.iterations // 8) == 0:
            print(f"iteration {i + 1}: log density {logp:.0f}, {accepted} accepted")
    often = torch.arange(3, device="cuda")
    ids, logprobs, entropy = model.answers(t, w, often, n_top=3)
    for v in range(3):
        print(f"after word {v}: " + ", ".join(f"{int(i)} ({math.exp(float(p)):.2f})" for i, p in zip(ids[v], logprobs[v])) + f"; entropy {float(entropy[v]):.2f}")


if __name__ == "__main__":
    main()
