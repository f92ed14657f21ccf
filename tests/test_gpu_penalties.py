"""Logits adjusted by what was said before, biases and masks, and the gradient of that, against 64 bits."""
import math

import pytest
import torch

import categorical_ref as R
import learning_ref as L
import paper_1910_11141_amd as nuts

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed=1):
    return torch.Generator(device="cuda").manual_seed(seed)


def matrix(n, classes, dtype, g, pad=0, std=3.0, offset=0):
    flat = (torch.randn(n * (classes + pad) + offset, generator=g, device="cuda") * std).to(dtype)
    return flat[offset:].view(n, classes + pad)[:, :classes]


def history_of(n, length, classes, g, ids=torch.int64):
    """Some classes again and again, others once, pads and ids beyond the classes among them."""
    often = torch.randint(0, max(1, classes // 50), (n, length), generator=g, device="cuda")
    any_ = torch.randint(-3, classes + 3, (n, length), generator=g, device="cuda")
    return torch.where(torch.rand(n, length, generator=g, device="cuda") < 0.6, often, any_).to(ids)


def rows(n, low, high, g):
    return torch.rand(n, generator=g, device="cuda") * (high - low) + low


def places(n, most, g):
    return torch.randint(-1, most + 3, (n,), generator=g, device="cuda").int()


def masks(n, classes, g, one=False):
    mask = torch.rand(1 if one else n, classes, generator=g, device="cuda") < 0.7
    if not one and n > 1:
        mask[1] = False  # a row in which nothing may come
    return R.pack_bits(mask[0] if one else mask)


def check(logits, history, **kw):
    want, bound = L.penalties(logits, history, **kw)
    got = nuts.nuts_penalties(logits, history, **kw)
    assert got.shape == logits.shape and got.dtype == logits.dtype and got.stride(1) == 1
    assert L.close(got, want, bound)
    # in place the same bits
    there = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device="cuda").copy_(logits)
    assert nuts.nuts_penalties(there, history, out=there, **kw) is there
    assert torch.equal(there.nan_to_num(nan=77.0), got.nan_to_num(nan=77.0))
    return got


SIZES = [(1, 1, 1), (1, 7, 3), (3, 33, 40), (5, 8191, 17), (2, 8192, 600), (4, 8193, 1), (3, 16385, 5000), (7, 1000, 10), (2, 40001, 20000)]


@pytest.mark.parametrize("n,classes,length", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_all_of_it(n, classes, length, dtype):
    g = gen(n + classes)
    check(matrix(n, classes, dtype, g, pad=classes % 5), history_of(n, length, classes, g), lengths=places(n, length, g), prompts=places(n, length, g),
          repetition=rows(n, 0.5, 2.0, g), frequency=rows(n, -0.5, 1.0, g), presence=rows(n, -1.0, 1.0, g), bias=torch.randn(classes, generator=g, device="cuda"),
          bias_ids=torch.randint(-2, classes + 2, (n, 9), generator=g, device="cuda"), bias_values=torch.randn(n, 9, generator=g, device="cuda"),
          allowed=masks(n, classes, g))


@pytest.mark.parametrize("which", ["history", "prompts", "repetition", "frequency", "bias", "rows of biases", "some biases", "mask", "one mask", "nothing"])
@pytest.mark.parametrize("dtype,ids", [(F32, torch.int32), (BF16, torch.int64), (F16, torch.int32)])
def test_each_by_itself(which, dtype, ids):
    n, classes, length = 6, 9001, 300
    g = gen(3)
    logits, history = matrix(n, classes, dtype, g, pad=3, offset=1), history_of(n, length, classes, g, ids)
    if which == "history":
        check(logits, history, repetition=1.3, frequency=0.25, presence=-0.5)
    elif which == "prompts":
        check(logits, history, lengths=places(n, length, g), prompts=places(n, length, g), frequency=0.5, presence=0.125)
    elif which == "repetition":
        check(logits, history, repetition=rows(n, 0.5, 2.0, g))
    elif which == "frequency":
        check(logits, history, frequency=rows(n, -1.0, 1.0, g))
    elif which == "bias":
        check(logits, None, bias=torch.randn(1, classes, generator=g, device="cuda"))
    elif which == "rows of biases":
        check(logits, None, bias=torch.randn(n, classes + 2, generator=g, device="cuda")[:, :classes])
    elif which == "some biases":
        check(logits, history, repetition=1.5, bias_ids=history[:, :40], bias_values=torch.randn(n, 40, generator=g, device="cuda"))
    elif which == "mask":
        check(logits, None, allowed=masks(n, classes, g))
    elif which == "one mask":
        check(logits, history, presence=2.0, allowed=masks(n, classes, g, one=True))
    else:
        assert torch.equal(check(logits, history), logits)
        assert torch.equal(check(logits, None), logits)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_text_of_which_each_row_has_seen_the_beginning(dtype):
    n, classes, g = 300, 8200, gen(4)
    text = history_of(1, n, classes, g, torch.int32)[0]
    lengths = torch.arange(n, device="cuda").int()
    kw = dict(lengths=lengths, repetition=1.2, frequency=0.1, presence=0.3)
    got = check(matrix(n, classes, dtype, g), text, **kw)
    logits = matrix(n, classes, dtype, gen(5))
    assert torch.equal(nuts.nuts_penalties(logits, text, **kw), nuts.nuts_penalties(logits, text.expand(n, -1).contiguous(), **kw))
    assert got.shape == (n, classes)
    # lengths that rise, fall and stay, prompts that do, too
    for order in (torch.arange(n - 1, -1, -1), torch.randperm(n, generator=torch.Generator().manual_seed(1)), torch.arange(n) // 7):
        lengths = order.to("cuda").int()
        for prompts in (None, lengths // 3, (n - lengths) // 2, torch.full_like(lengths, 50)):
            check(logits, text, lengths=lengths, prompts=prompts, repetition=rows(n, 1.0, 2.0, g), frequency=rows(n, 0.0, 1.0, g), presence=0.5)
        # biases of single classes, each row's its own, among classes that were said and others
        ids = history_of(n, 11, classes, g, torch.int32)
        check(logits, text, lengths=lengths, repetition=1.5, bias_ids=ids, bias_values=torch.randn(n, 11, generator=g, device="cuda"))


def test_more_rows_of_one_text_than_workgroups_at_a_time():
    n, classes, g = 2500, 300, gen(21)
    text = history_of(1, 700, classes, g)
    lengths = (torch.arange(n, device="cuda") * 700 // n).int()
    ids = history_of(n, 3, classes, g)
    check(matrix(n, classes, BF16, g), text, lengths=lengths, prompts=lengths // 2, repetition=1.25, frequency=0.125,
          bias_ids=ids, bias_values=torch.randn(n, 3, generator=g, device="cuda"), allowed=masks(n, classes, g))


def test_a_class_said_very_often():
    """Counts beyond 16 bits, and one counter that all threads add to."""
    classes, length = 20, 200000
    history = torch.full((2, length), 7, device="cuda")
    history[1, ::2] = 3
    logits = matrix(2, classes, F32, gen())
    check(logits, history, frequency=2.0 ** -12, prompts=torch.tensor([1000, 0], device="cuda").int())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_what_is_not_finite(dtype):
    n, classes, g = 4, 300, gen(6)
    logits = matrix(n, classes, dtype, g)
    low = torch.finfo(dtype).min
    for i, x in enumerate((math.nan, math.inf, -math.inf, low, -low, 0.0, -0.0)):
        logits[:, i] = x
    history = torch.arange(0, 20, 2, device="cuda").expand(n, -1)
    kw = dict(repetition=2.0, frequency=1.0, presence=1.0)
    check(logits, history, **kw)
    check(logits, history + 1, **kw)
    bias = torch.zeros(classes, device="cuda")
    bias[20], bias[21] = -math.inf, math.nan
    check(logits, history, bias=bias, **kw)
    got = check(logits, history, bias=bias, allowed=torch.zeros(10, dtype=torch.int32, device="cuda"), **kw)
    assert bool((got == -math.inf).all())
    ids = torch.tensor([[20, 21, 0, 5]], device="cuda").expand(n, -1)
    check(logits, history, bias_ids=ids, bias_values=torch.tensor([[-math.inf, math.nan, 1.0, 2.0]], device="cuda").expand(n, -1), **kw)


def test_biases_of_the_same_class_add_up_in_their_order():
    g = gen(7)
    logits = torch.zeros(1, 50, device="cuda")
    for n_bias in (1, 2, 1024):
        ids = torch.full((1, n_bias), 9, device="cuda")
        ids[0, n_bias // 2:] = 11
        values = torch.randn(1, n_bias, generator=g, device="cuda") * 10.0 ** torch.randint(-4, 5, (1, n_bias), generator=g, device="cuda")
        got = nuts.nuts_penalties(logits, bias_ids=ids, bias_values=values)
        for v, some in ((9, values[0, :n_bias // 2]), (11, values[0, n_bias // 2:])):
            want = torch.zeros(())
            for i, x in enumerate(some.cpu()):
                want = x if i == 0 else want + x
            assert float(got[0, v]) == float(want)


def test_places_that_do_not_change_are_not_written():
    """Between rows, and in place."""
    g = gen(8)
    flat = torch.full((3, 9000), 5.0, dtype=BF16, device="cuda")
    out = flat[:, :8500]
    logits = matrix(3, 8500, BF16, g)
    nuts.nuts_penalties(logits, torch.tensor([1, 8499], device="cuda"), repetition=1.5, out=out)
    assert bool((flat[:, 8500:] == 5.0).all()) and bool((flat[:, :8500] != 5.0).any())


def test_long_rows_and_strides_beyond_32_bits():
    n, stride = 5, (1 << 30) + 7
    flat = torch.empty(4 * stride + 20000, dtype=BF16, device="cuda")
    logits = torch.as_strided(flat, (n, 20000), (stride, 1))
    g = gen(9)
    logits.copy_(matrix(n, 20000, BF16, g))
    before = logits.contiguous()
    history = history_of(n, 50, 20000, g)
    want, bound = L.penalties(before, history, repetition=1.5, presence=1.0)
    nuts.nuts_penalties(logits, history, repetition=1.5, presence=1.0, out=logits)
    assert L.close(logits.contiguous(), want, bound)
    logits = matrix(2, 300_001, F32, g)
    check(logits, history_of(2, 100, 300_001, g), repetition=1.1, frequency=0.2)


def test_histories_of_other_orders():
    g = gen(10)
    logits = matrix(3, 500, F32, g)
    history = history_of(40, 3, 500, g).t()
    check(logits, history, repetition=1.5)
    windows = torch.as_strided(history_of(1, 60, 500, g), (3, 40), (1, 1))   # rows that overlap
    check(logits, windows, repetition=1.5, frequency=1.0)
    check(logits, history_of(3, 0, 500, g), repetition=1.5)
    assert nuts.nuts_penalties(logits[:0], history[:0]).shape == (0, 500)


@pytest.mark.parametrize("dtype,length", [(BF16, 40), (F16, 20000), (F32, 2048), (F32, 17001)])
@pytest.mark.parametrize("n_bias", [0, 5, 1024])
def test_wide_slices(dtype, length, n_bias):
    """Histories of their own of enough rows of enough classes: three slices of 16384, the last of which is nearly empty."""
    n, classes, g = 90, 32771, gen(22)
    kw = {}
    if n_bias:
        kw = dict(bias_ids=torch.randint(-2, classes + 2, (n, n_bias), generator=g, device="cuda"), bias_values=torch.randn(n, n_bias, generator=g, device="cuda"))
        kw["bias_ids"][:, n_bias // 2] = kw["bias_ids"][:, 0]
        kw["bias_ids"][3] = 32770
    check(matrix(n, classes, dtype, g, pad=1), history_of(n, length, classes, g), lengths=places(n, length, g), prompts=places(n, length, g),
          repetition=rows(n, 0.5, 2.0, g), frequency=rows(n, 0.0, 0.25, g), presence=0.5, bias=torch.randn(classes, generator=g, device="cuda"),
          allowed=masks(n, classes, g), **kw)
    check(matrix(n, classes, dtype, g), history_of(n, length, classes, g, torch.int32), repetition=1.5, presence=1.0, **kw)


def test_outputs_past_the_caches():
    n, classes, g = 2100, 32003, gen(23)
    logits = matrix(n, classes, BF16, g)
    text = history_of(1, n, classes, g, torch.int32)[0]
    check(logits, text, lengths=torch.arange(n, device="cuda").int(), repetition=1.5, frequency=0.25)
    check_grad(logits, logits.flip(0), text, lengths=torch.arange(n, device="cuda").int(), repetition=1.5)


def test_ids_of_two_types():
    """A bias of a class that only 64 bits tell from one of the table's."""
    g = gen(24)
    logits, history = matrix(2, 100, F32, g), history_of(2, 30, 100, g, torch.int32)
    ids = torch.tensor([[5, 2 ** 32 + 7, -2 ** 32 + 9], [2 ** 31 + 3, 11, 11]], device="cuda")
    check(logits, history, repetition=1.5, bias_ids=ids, bias_values=torch.ones(2, 3, device="cuda"))
    check(logits, history[0], repetition=1.5, bias_ids=ids, bias_values=torch.ones(2, 3, device="cuda"))
    check(logits, history.long() + 2 ** 33 * (history.long() % 3), presence=1.5, bias_ids=ids.int().clamp(0, 50), bias_values=torch.ones(2, 3, device="cuda"))


# ---- gradient -----------------------------------------------------------------------------------------------------------

def check_grad(grad, logits, history, **kw):
    want, bound, want_bias, bias_bound = L.penalties_grad(grad, logits, history, **kw)
    got, bias = nuts.nuts_penalties_grad(grad, logits, history, want_bias=True, **kw)
    assert got.dtype == grad.dtype and bias.dtype == F32
    assert L.close(got, want, bound) and L.close(bias, want_bias, bias_bound)
    alone, none = nuts.nuts_penalties_grad(grad, logits, history, **kw)
    assert none is None and torch.equal(alone, got)
    none, alone = nuts.nuts_penalties_grad(grad, logits, history, want_logits=False, want_bias=True, **kw)
    assert none is None and L.close(alone, want_bias, bias_bound)
    there = torch.empty_strided(grad.shape, grad.stride(), dtype=grad.dtype, device="cuda").copy_(grad)
    again, bias_again = nuts.nuts_penalties_grad(there, logits, history, want_bias=True, out=there, **kw)
    assert again is there and torch.equal(there, got) and torch.equal(bias_again, bias)
    there.copy_(grad)
    nuts.nuts_penalties_grad(there, logits, history, out=there, **kw)
    assert torch.equal(there, got)


@pytest.mark.parametrize("n,classes,length", SIZES + [(1500, 1000, 10), (5000, 130, 3), (2100, 9000, 2)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_grad(n, classes, length, dtype):
    g = gen(n + classes)
    check_grad(matrix(n, classes, dtype, g, pad=classes % 3, std=0.1), matrix(n, classes, dtype, g, pad=classes % 5), history_of(n, length, classes, g),
               lengths=places(n, length, g), repetition=rows(n, 0.5, 2.0, g), allowed=masks(n, classes, g) if n % 2 else masks(n, classes, g, one=True))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grad_of_one_text(dtype):
    n, classes, g = 1300, 8300, gen(11)
    text = history_of(1, n, classes, g)
    for lengths in (torch.arange(n), torch.arange(n - 1, -1, -1), torch.arange(n) // 9 * 5 % 700):
        check_grad(matrix(n, classes, dtype, g), matrix(n, classes, dtype, g), text, lengths=lengths.to("cuda").int(), repetition=1.25)
    check_grad(matrix(n, classes, dtype, g), matrix(n, classes, dtype, g), None)


def test_grad_of_no_rows_is_zero():
    x = torch.zeros(0, 70, device="cuda")
    grad, bias = nuts.nuts_penalties_grad(x, x, None, want_bias=True)
    assert grad.shape == (0, 70) and bool((bias == 0).all())


def test_grad_where_something_is_not_finite():
    n, classes, g = 3, 200, gen(12)
    logits, grad = matrix(n, classes, F32, g), matrix(n, classes, F32, g)
    for i, x in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0)):
        logits[:, i] = x
        grad[:, 10 + i] = x
    mask = torch.ones(classes, dtype=torch.bool, device="cuda")
    mask[10:13] = False
    history = torch.arange(0, 14, 1, device="cuda")
    want, bound, want_bias, bias_bound = L.penalties_grad(grad, logits, history, repetition=1.5, allowed=R.pack_bits(mask))
    got, bias = nuts.nuts_penalties_grad(grad, logits, history, repetition=1.5, allowed=R.pack_bits(mask), want_bias=True)
    assert L.close(got, want, bound) and L.close(bias, want_bias, bias_bound)
    assert bool((got[:, 10:13] == 0).all()) and bool((bias[10:13] == 0).all())


def test_grad_against_differences():
    """In 32 bits with inputs of few bits: what z changes by over steps of 2^-6 is exact but for the division."""
    n, classes, g = 4, 700, gen(13)
    logits = (torch.randint(-63, 64, (n, classes), generator=g, device="cuda") * 2 + 1) / 16.0   # (none is 0, and none changes its sign)
    grad = torch.randint(-8, 9, (n, classes), generator=g, device="cuda").float()
    history, bias = history_of(n, 90, classes, g), torch.randint(-8, 9, (classes,), generator=g, device="cuda").float()
    kw = dict(repetition=1.5, frequency=0.25, presence=0.5)
    dx, db = nuts.nuts_penalties_grad(grad, logits, history, repetition=1.5, want_bias=True)
    h = 2.0 ** -6
    z = lambda x, b: nuts.nuts_penalties(x, history, bias=b, **kw).double()  # noqa: E731
    slope = (z(logits + h, bias) - z(logits - h, bias)) / (2 * h)
    most = 32.0  # |z| at most: each z is off by three roundings of it, and the difference by two such
    assert float((slope * grad - dx).abs().max()) <= 8 * 6 * most * 2.0 ** -24 / (2 * h)
    total = ((z(logits, bias + h) - z(logits, bias - h)) / (2 * h) * grad).sum(0)
    assert float((total - db).abs().max()) <= n * 8 * 6 * most * 2.0 ** -24 / (2 * h)


# ---- how they are called ------------------------------------------------------------------------------------------------

def test_calls_repeated_captured_and_on_other_streams():
    n, classes, g = 9, 20011, gen(14)
    logits, grad = matrix(n, classes, BF16, g), matrix(n, classes, BF16, g)
    kw = dict(lengths=places(n, 400, g), repetition=rows(n, 1.0, 2.0, g), allowed=masks(n, classes, g))
    history = history_of(n, 400, classes, g)
    more = dict(frequency=0.5, presence=0.1, bias=torch.randn(classes, generator=g, device="cuda"))

    def both():
        return nuts.nuts_penalties(logits, history, **kw, **more), *nuts.nuts_penalties_grad(grad, logits, history, want_bias=True, **kw)

    want = [t.clone() for t in both()]
    assert all(torch.equal(a, b) for a, b in zip(both(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for k in range(4):
        logits.copy_(matrix(n, classes, BF16, gen(20 + k)))
        kw["lengths"].copy_(places(n, 400, gen(30 + k)))
        want = both()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # on a stream of the library's own
    nuts.nuts_set_stream(side)
    try:
        got = both()
    finally:
        nuts.nuts_set_stream(None)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
