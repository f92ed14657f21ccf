"""AdamW at the ends of binary32's range: a v whose root has to be found though v is below 2^-126, denominators of which the reciprocal is not a usual
number.  Gradients are 0 and the moments shrink by a half (which is exact), so that what the update divides is known to the last bit."""
import math

import pytest
import torch

import learning_ref as L
import paper_1910_11141_amd as nuts

pytestmark = pytest.mark.gpu

U = L.U
HALF = dict(betas=(0.5, 0.5), weight_decay=0.0, step=1)   # m / (1 - 0.5) and v / (1 - 0.5) divide by a half


def updates(m, v, lr, eps):
    """One step of parameters 0 from moments 2 m and 2 v with gradients of 0, and its update in 64 bits."""
    p, m2, v2 = torch.zeros_like(m), 2 * m, 2 * v
    moments = nuts.Moments([p], states=([m2], [v2]))
    nuts.nuts_adamw(moments, [torch.zeros_like(m)], lr=lr, eps=eps, **HALF)
    assert torch.equal(m2, m) and torch.equal(v2, v)
    return p, -2 * lr * m.double() / (torch.sqrt(2 * v.double()) + eps)


@pytest.mark.parametrize("n", [1, 255, 3000])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -133, 2.0 ** -110, 2.0 ** -90, 1e-25, 2.0 ** -64])
@pytest.mark.parametrize("largest", [2 ** 6, 2 ** 22, 2 ** 30])
def test_roots_of_what_is_below_the_usual_numbers(n, eps, largest):
    """v of 1 to `largest` times 2^-149, in the same waves as v of 1.  Off by a unit in the last place for the root and for the reciprocal (two halves
    each), and half of one for the root's factor, denominator, step's size, product and sum each: 9 U, and what these add to each other."""
    g = torch.Generator(device="cuda").manual_seed(n)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    k = torch.randint(1, largest + 1, (n,), generator=g, device="cuda")
    if largest > 2 ** 24:
        k = k // 64 * 64 + 64   # (24 places)
    v = (k.double() * 2.0 ** -149).float()
    v[5::7] = 1.0
    m = (torch.rand(n, generator=g, device="cuda") + 1) * torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -1.0, 1.0) * 2.0 ** -70
    got, want = updates(m, v, 2.0 ** -9, eps)
    assert bool(((got.double() - want).abs() <= 10 * U * want.abs()).all())


@pytest.mark.parametrize("eps,m,v,lr", [
    (2.0 ** -133, 2.0 ** -140, 0.0, 2.0 ** -9),          # the denominator is eps, which is below the usual numbers, and so is m
    (2.0 ** -127, 2.0 ** -100, 0.0, 2.0 ** -9),
    (2.0 ** -149, -2.0 ** -149, 0.0, 2.0 ** -9),
    (1.5 * 2.0 ** 126, 2.0 ** 60, 1.0, 2.0 ** 60),       # the reciprocal is below them
    (1.5 * 2.0 ** 127, -2.0 ** 61, 2.0 ** 100, 2.0 ** 60),
    (2.0 ** -99, 2.0 ** -50, 2.0 ** -126, 2.0 ** -9), (2.0 ** -101, 2.0 ** -50, 2.0 ** -126, 2.0 ** -9),   # either way to divide
    (2.0 ** 99, 2.0 ** 50, 2.0 ** 126, 2.0 ** 9), (2.0 ** 101, 2.0 ** 50, 2.0 ** 126, 2.0 ** 9),
    (0.0, 2.0 ** -30, 2.0 ** 126, 2.0 ** -9), (0.0, 2.0 ** 40, 2.0 ** 90, 2.0 ** -9), (0.0, 2.0 ** -75, 2.0 ** -149, 2.0 ** -9),
])
@pytest.mark.parametrize("n", [1, 700])
def test_denominators_beyond_the_usual_numbers(eps, m, v, lr, n):
    got, want = updates(torch.full((n,), m, device="cuda"), torch.full((n,), v, device="cuda"), lr, eps)
    assert bool((want != 0).all()) and bool(((got.double() - want).abs() <= 10 * U * want.abs()).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("params", [torch.float32, torch.bfloat16])
def test_moments_of_zero_and_a_denominator_below_the_usual_numbers(bits, params):
    """0 / eps is 0; 0 / 0 is not a number."""
    p = torch.ones(600, dtype=params, device="cuda")
    moments = nuts.Moments([p], bits=bits)
    for eps in (2.0 ** -149, 2.0 ** -133, 2.0 ** -127):
        nuts.nuts_adamw(moments, [torch.zeros_like(p)], step=1, lr=0.1, eps=eps, weight_decay=0.0)
        assert bool((p == 1).all())
    nuts.nuts_adamw(moments, [torch.zeros_like(p)], step=1, lr=0.1, eps=0.0, weight_decay=0.0)
    assert bool(p.isnan().all())


def test_a_first_step_with_gradients_whose_squares_are_below_the_usual_numbers():
    """The sign of the gradient, times the rate: (1 - beta) g / (1 - beta) / sqrt((1 - beta) g^2 / (1 - beta)).  v is rounded to a multiple of 2^-149
    twice, g^2 and its product, which moves v by 1.001 times half of that."""
    g = torch.tensor([1e-17, -3e-18, 1e-18, -3e-19, 1e-19, 3e-20], device="cuda").repeat(100)
    p = torch.zeros_like(g)
    nuts.nuts_adamw(nuts.Moments([p]), [g], step=1, lr=0.5, eps=0.0, weight_decay=0.0)
    off = 1.001 * 2.0 ** -150 / (0.001 * g.double() ** 2)
    low, high = 0.5 / (1 + off).sqrt() * (1 - 20 * U), 0.5 / (1 - off).sqrt() * (1 + 20 * U)
    got = p.double() * -torch.sign(g.double())
    assert bool((off < 0.6).all()) and bool(((got >= low) & (got <= high)).all())


@pytest.mark.parametrize("top", [2.0 ** -64, 2.0 ** -70, 1e-15])
def test_codes_of_a_v_below_the_usual_numbers(top):
    """A block whose largest v is top^2: a v above 0 has a code, one of the two beside it, as a larger one would have."""
    n = 5 * 256 + 77
    g = torch.Generator(device="cuda").manual_seed(3)
    codes = torch.randint(0, 255, (n,), generator=g, device="cuda").to(torch.uint8)
    codes[::256] = 254
    codes[1::256] = 0
    blocks = -(-n // 256)
    zeros = torch.zeros(blocks, device="cuda")
    states = ([torch.zeros(n, dtype=torch.int8, device="cuda")], [codes], [zeros], [torch.full((blocks,), top / 254 ** 2, device="cuda")])
    v = L.v_values(codes, states[3][0])
    p = torch.zeros(n, device="cuda")
    moments = nuts.Moments([p], bits=8, states=states)
    nuts.nuts_adamw(moments, [torch.zeros(n, device="cuda")], lr=0.1, eps=1e-8, seed=11, **HALF)
    new = v / 2
    # the value of a code is three roundings of its root and one of the square, which below 2^-126 is to a multiple of 2^-149; its half is another such
    bound = 4 * U * v + 2.0 ** -150 * 1.51
    low, high = (new - bound).clamp(min=0).sqrt() * (1 - 4 * U), (new + bound).sqrt() * (1 + 4 * U)
    largest_low, largest_high = L.block_max(low), L.block_max(high)
    scale = states[3][0].double()
    assert bool(((scale >= largest_low / 254 ** 2 * (1 - 3 * U)) & (scale <= largest_high / 254 ** 2 * (1 + 3 * U))).all())
    scale = scale.repeat_interleave(256)[:n]
    u = ((L.words(n, 11, 1, 0, "cuda") >> 10 & 1023) + 0.5) / 1024
    x_low, x_high = low / scale, high / scale
    off = 32 * U * (x_high + 1)
    got = codes.double()
    least = torch.where(low > 0, torch.maximum(x_low - off, torch.full_like(low, 1e-30)), 0.0)
    most = torch.where(v == 0, 0.0, x_high + off)
    assert bool(((got >= L.v_codes(least.sqrt(), u)) & (got <= L.v_codes(most.sqrt(), u))).all())
    assert bool((got[low > 0] >= 1).all()) and bool((got[v == 0] == 0).all()) and int((low > 0).sum()) > n // 2 and bool((p == 0).all())
