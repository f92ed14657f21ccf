"""Penalties, norms and AdamW steps refuse what they cannot do, on the host and before anything is written."""
import copy
import ctypes as C
import subprocess
import sys

import pytest
import torch

import learning_ref as L
from paper_1910_11141_amd import binding as B
import paper_1910_11141_amd as nuts

P = C.c_void_p(4096)   # (never followed: a call that would has been refused)
Q = C.c_void_p(8192)


def penalties(**kw):
    d = dict(dtype=0, id_type=0, n_rows=4, n_classes=5, row_stride=8, out_stride=8, allowed_stride=0, bias_stride=0, history_len=6, history_stride=6, n_bias=2,
             repetition=1.0, frequency=0.0, presence=0.0)
    return C.byref(B.nuts_penalties_desc(**{**d, **kw}))


def adamw(**kw):
    d = dict(param_dtype=0, grad_dtype=0, copy_dtype=2, state_bits=32, lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, scale=1.0, step=1, seed=0)
    return C.byref(B.nuts_adamw_desc(**{**d, **kw}))


def table(kind, *entries):
    return (kind * len(entries))(*entries)


def tensor(**kw):
    d = dict(param=4096, grad=8192, copy=0, m=12288, v=16384, m_scale=20480, v_scale=24576, n=5)
    return B.nuts_adamw_tensor(**{**d, **kw})


def refused(rc, word=None):
    assert rc == B.NUTS_E_INVALID_ARG
    assert word is None or word in B.nuts_last_error(), B.nuts_last_error()


def test_struct_layouts():
    assert (C.sizeof(B.nuts_penalties_desc), C.sizeof(B.nuts_tensor), C.sizeof(B.nuts_adamw_tensor), C.sizeof(B.nuts_adamw_desc)) == (104, 24, 64, 80)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad,word", [
    (dict(dtype=1), "dtype"), (dict(dtype=4), "dtype"), (dict(id_type=2), "id_type"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=2 ** 31 - 1), "n_rows"),
    (dict(n_classes=0), "n_classes"), (dict(n_classes=2 ** 31 - 2 ** 18, row_stride=2 ** 31, out_stride=2 ** 31), "n_classes"), (dict(row_stride=4), "row_stride"),
    (dict(row_stride=2 ** 61), "row_stride"), (dict(out_stride=4), "out_stride"), (dict(out_stride=2 ** 61), "out_stride"),
    (dict(n_classes=65, row_stride=65, out_stride=65, allowed_stride=2), "allowed_stride"), (dict(allowed_stride=-1), "allowed_stride"),
    (dict(allowed_stride=2 ** 61), "allowed_stride"), (dict(bias_stride=4), "bias_stride"), (dict(bias_stride=-8), "bias_stride"),
    (dict(bias_stride=2 ** 61), "bias_stride"), (dict(history_len=-1), "history_len"), (dict(history_len=2 ** 29, history_stride=2 ** 29), "history_len"),
    (dict(history_stride=5), "history_stride"), (dict(history_stride=-6), "history_stride"), (dict(history_stride=2 ** 61), "history_stride"),
    (dict(n_bias=-1), "n_bias"), (dict(n_bias=1025), "n_bias"), (dict(repetition=0.0), "repetition"), (dict(repetition=-1.0), "repetition"),
    (dict(repetition=NAN), "repetition"), (dict(repetition=INF), "repetition"), (dict(repetition=1e-60), "repetition"), (dict(frequency=NAN), "frequency"),
    (dict(presence=INF), "presence"), (dict(presence=1e300), "presence")])
def test_penalties_descriptors(bad, word):
    lib, n = B.lib(), C.c_int64()
    refused(lib.nuts_penalties(penalties(**bad), *[P] * 11, Q), word)
    refused(lib.nuts_penalties_grad(penalties(**bad), P, 8, Q, P, P, P, P, P, P, P, 1 << 40), word)
    refused(lib.nuts_penalties_grad_workspace(penalties(**bad), C.byref(n)), word)


def test_penalties_ends_of_the_ranges():
    lib, n = B.lib(), C.c_int64()
    wide = dict(n_rows=1, n_classes=2 ** 31 - 2 ** 18 - 1, row_stride=2 ** 31, out_stride=2 ** 31)
    for good in (wide, dict(n_rows=2 ** 31 - 2), dict(history_len=2 ** 29 - 1, history_stride=2 ** 29), dict(history_len=0, history_stride=0), dict(n_bias=1024)):
        assert lib.nuts_penalties_grad_workspace(penalties(**good), C.byref(n)) == B.NUTS_OK and n.value > 0, good


def test_penalties_pointers():
    lib, n = B.lib(), C.c_int64()
    refused(lib.nuts_penalties(None, *[P] * 12))
    refused(lib.nuts_penalties_grad(None, P, 8, P, P, P, P, P, P, P, P, 1 << 40))
    refused(lib.nuts_penalties_grad_workspace(None, C.byref(n)))
    refused(lib.nuts_penalties_grad_workspace(penalties(), None))
    refused(lib.nuts_penalties(penalties(), None, *[P] * 10, Q))
    refused(lib.nuts_penalties(penalties(), *[P] * 11, None))
    refused(lib.nuts_penalties(penalties(), P, None, *[P] * 9, Q), "history")
    refused(lib.nuts_penalties(penalties(), *[P] * 8, None, P, P, Q), "bias_ids")
    refused(lib.nuts_penalties(penalties(), *[P] * 9, None, P, Q), "bias_ids")
    refused(lib.nuts_penalties(penalties(out_stride=9), *[P] * 11, P), "in place")
    grad = lambda desc, g=P, gs=8, x=Q, h=P, dx=P, db=P, ws=P, size=1 << 40: lib.nuts_penalties_grad(desc, g, gs, x, h, P, P, P, dx, db, ws, size)  # noqa: E731
    refused(grad(penalties(), gs=4), "grad_stride")
    refused(grad(penalties(), gs=2 ** 61), "grad_stride")
    refused(grad(penalties(), g=None))
    refused(grad(penalties(), x=None))
    refused(grad(penalties(), h=None), "history")
    refused(grad(penalties(), dx=Q), "overlap")
    refused(grad(penalties(out_stride=9)), "in place")
    assert lib.nuts_penalties_grad_workspace(penalties(), C.byref(n)) == B.NUTS_OK
    refused(grad(penalties(), size=n.value - 1), "workspace")
    refused(grad(penalties(), ws=None), "workspace")
    refused(grad(penalties(), ws=C.c_void_p(4097)), "aligned")


@pytest.mark.parametrize("bad,word", [
    (dict(param_dtype=3), "param_dtype"), (dict(param_dtype=1), "param_dtype"), (dict(grad_dtype=1), "grad_dtype"), (dict(copy_dtype=0), "copy_dtype"),
    (dict(state_bits=16), "state_bits"), (dict(lr=NAN), "lr"), (dict(lr=INF), "lr"), (dict(beta1=1.0), "beta1"), (dict(beta1=-0.1), "beta1"), (dict(beta2=1.0), "beta2"),
    (dict(beta2=1.0 - 1e-12), "beta2"), (dict(beta2=NAN), "beta2"), (dict(eps=-1e-8), "eps"), (dict(eps=NAN), "eps"), (dict(eps=1e300), "eps"),
    (dict(weight_decay=NAN), "weight_decay"), (dict(scale=INF), "scale"), (dict(step=0), "step"), (dict(step=-5), "step")])
def test_adamw_descriptors(bad, word):
    refused(B.lib().nuts_adamw(adamw(**bad), table(B.nuts_adamw_tensor, tensor()), 1, None, None, None), word)


def test_tables_of_tensors():
    lib, n = B.lib(), C.c_int64()
    one = table(B.nuts_adamw_tensor, tensor())
    refused(lib.nuts_adamw(None, one, 1, None, None, None))
    for call in (lambda t, k: lib.nuts_adamw(adamw(), t, k, None, None, None), lambda t, k: lib.nuts_adamw_values(t, k, 0)):
        refused(call(None, 1), "tensors")
        refused(call(one, -1), "n_tensors")
        refused(call(one, 2 ** 20 + 1), "n_tensors")
        for bad in (dict(n=-1), dict(n=2 ** 40 + 1)):
            refused(call(table(B.nuts_adamw_tensor, tensor(), tensor(**bad)), 2), "tensor 1")
        for bad in (dict(m=0), dict(v=0)):
            refused(call(table(B.nuts_adamw_tensor, tensor(), tensor(**bad)), 2), "tensor 1")
        assert call(None, 0) == B.NUTS_OK
        assert call(table(B.nuts_adamw_tensor, tensor(n=0, m=0), tensor(param=0, grad=0)), 2) == B.NUTS_OK
    refused(lib.nuts_adamw(adamw(), table(B.nuts_adamw_tensor, tensor(param=0)), 1, None, None, None), "tensor 0")
    for bad in (dict(m_scale=0), dict(v_scale=0)):
        refused(lib.nuts_adamw(adamw(state_bits=8), table(B.nuts_adamw_tensor, tensor(**bad)), 1, None, None, None), "tensor 0")
        refused(lib.nuts_adamw_values(table(B.nuts_adamw_tensor, tensor(**bad)), 1, 0), "tensor 0")
    refused(lib.nuts_adamw_values(one, 1, 1), "dtype")
    some = lambda **kw: table(B.nuts_tensor, B.nuts_tensor(**{**dict(data=4096, n=100000, dtype=0, reserved=0), **kw}))  # noqa: E731
    norm = lambda t, k=1, most=1.0, ws=P, size=1 << 30: lib.nuts_norm(t, k, most, P, P, ws, size)  # noqa: E731
    for bad, word in ((dict(data=None), "data"), (dict(n=-1), "n of"), (dict(n=2 ** 40 + 1), "n of"), (dict(dtype=1), "dtype")):
        refused(norm(some(**bad)), word)
        refused(lib.nuts_norm_workspace(some(**bad), 1, C.byref(n)), word)
    refused(norm(None), "tensors")
    refused(norm(some(), k=-1), "n_tensors")
    half = [B.nuts_tensor(4096, 2 ** 39 + 1, 2, 0)] * 2
    refused(norm(table(B.nuts_tensor, *half), k=2), "2^40")
    for most in (0.0, -1.0, NAN, INF):
        refused(norm(some(), most=most), "max_norm")
    refused(lib.nuts_norm_workspace(some(), 1, None))
    assert lib.nuts_norm_workspace(some(), 1, C.byref(n)) == B.NUTS_OK and n.value > 0
    refused(norm(some(), size=n.value - 1), "workspace")
    refused(norm(some(), ws=None), "workspace")
    refused(norm(some(), ws=C.c_void_p(4097)), "aligned")
    assert lib.nuts_norm(some(), 1, 1.0, None, None, P, n.value) == B.NUTS_OK   # nothing is asked for


def test_nothing_to_do_is_no_error():
    lib, n = B.lib(), C.c_int64()
    assert lib.nuts_penalties(penalties(n_rows=0), *[None] * 12) == B.NUTS_OK
    assert lib.nuts_penalties_grad(penalties(n_rows=0), None, 8, None, None, None, None, None, P, None, None, 0) == B.NUTS_OK
    assert lib.nuts_penalties_grad(penalties(), P, 8, Q, P, P, P, P, None, None, None, 0) == B.NUTS_OK
    assert lib.nuts_penalties_grad_workspace(penalties(n_rows=0), C.byref(n)) == B.NUTS_OK and n.value == 0


def test_tensors_that_do_not_fit():
    x, ids, i32, f = torch.zeros(4, 8), torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 3)
    for call in (lambda: nuts.nuts_penalties(x.double()), lambda: nuts.nuts_penalties(x.t()), lambda: nuts.nuts_penalties(x, ids.float()),
                 lambda: nuts.nuts_penalties(x, ids[:3]), lambda: nuts.nuts_penalties(x, ids[None]), lambda: nuts.nuts_penalties(x, ids, lengths=i32.long()),
                 lambda: nuts.nuts_penalties(x, ids, lengths=i32[:3]), lambda: nuts.nuts_penalties(x, ids, prompts=i32[:3]),
                 lambda: nuts.nuts_penalties(x, ids, repetition=torch.ones(3)), lambda: nuts.nuts_penalties(x, ids, frequency=torch.ones(4).double()),
                 lambda: nuts.nuts_penalties(x, bias=torch.zeros(7)), lambda: nuts.nuts_penalties(x, bias=torch.zeros(3, 8)),
                 lambda: nuts.nuts_penalties(x, bias=torch.zeros(8).half()), lambda: nuts.nuts_penalties(x, bias=torch.zeros(8, 4).t()),
                 lambda: nuts.nuts_penalties(x, bias_ids=ids), lambda: nuts.nuts_penalties(x, bias_values=f),
                 lambda: nuts.nuts_penalties(x, bias_ids=ids, bias_values=f[:, :2]), lambda: nuts.nuts_penalties(x, bias_ids=ids[:3], bias_values=f[:3]),
                 lambda: nuts.nuts_penalties(x, bias_ids=ids, bias_values=f.half()), lambda: nuts.nuts_penalties(x, allowed=torch.zeros(2, dtype=torch.int32)),
                 lambda: nuts.nuts_penalties(x, out=torch.zeros(4, 7)), lambda: nuts.nuts_penalties(x, out=x.half()),
                 lambda: nuts.nuts_penalties_grad(x.half(), x), lambda: nuts.nuts_penalties_grad(x[:, :7], x), lambda: nuts.nuts_penalties_grad(x, x, ids[:2]),
                 lambda: nuts.nuts_penalties_grad(x, x, out=x, want_logits=False), lambda: nuts.nuts_penalties_grad(x, x, out=torch.zeros(3, 8)),
                 lambda: nuts.nuts_norm([]), lambda: nuts.nuts_norm([x, x.double()]),
                 lambda: nuts.Moments([]), lambda: nuts.Moments([x], bits=16), lambda: nuts.Moments([x.half()]), lambda: nuts.Moments([x, x.bfloat16()]),
                 lambda: nuts.Moments([x.t()]), lambda: nuts.Moments([x], copies=[]), lambda: nuts.Moments([x], copies=[x.clone()]),
                 lambda: nuts.Moments([x], copies=[x.half()[:3]]), lambda: nuts.Moments([x, x]), lambda: nuts.Moments([x[:3], x[2:]]),
                 lambda: nuts.Moments([x], states=([x.clone()], [x])), lambda: nuts.Moments([x], states=([x.clone()],)), lambda: nuts.Moments([x], states=([None], [x.clone()])),
                 lambda: nuts.Moments([x], bits=8, states=([x.char()], [x.byte()], [None], [torch.zeros(1)])),
                 lambda: nuts.Moments([x], states=([x.clone()], [x.clone().half()])), lambda: nuts.Moments([x], bits=8, states=([x.clone()], [x.clone()])),
                 lambda: nuts.Moments([x], bits=8, states=([x.clone().char()], [x.clone().byte()], [torch.zeros(2)], [torch.zeros(1)])),
                 lambda: nuts.nuts_adamw_values(nuts.Moments([x])), lambda: nuts.nuts_adamw_values(nuts.Moments([x], bits=8), out=([x], [])),
                 lambda: nuts.nuts_adamw_values(nuts.Moments([x], bits=8), out=([x.clone()], [x.half()])),
                 lambda: nuts.nuts_adamw_values(nuts.Moments([x], bits=8), dtype=torch.float64)):
        with pytest.raises(ValueError):
            call()
    mo = nuts.Moments([x, x[:2].clone()])
    g = [x.clone(), x[:2].clone()]
    for call in (lambda: nuts.nuts_adamw(mo, g[:1], step=1, lr=0.1), lambda: nuts.nuts_adamw(mo, [g[0], g[1].half()], step=1, lr=0.1),
                 lambda: nuts.nuts_adamw(mo, [g[0], g[1].view(-1)], step=1, lr=0.1), lambda: nuts.nuts_adamw(mo, [t.double() for t in g], step=1, lr=0.1),
                 lambda: nuts.nuts_adamw(mo, g, step=torch.ones(1), lr=0.1), lambda: nuts.nuts_adamw(mo, g, step=1, lr=torch.zeros(2)),
                 lambda: nuts.nuts_adamw(mo, g, step=1, lr=torch.zeros(1).double()), lambda: nuts.nuts_adamw(mo, g, step=1, lr=0.1, factor=torch.zeros(2))):
        with pytest.raises(ValueError):
            call()
    mo.params[0].data = torch.zeros(3, 8)
    with pytest.raises(ValueError):
        nuts.nuts_adamw(mo, [torch.zeros(3, 8), g[1]], step=1, lr=0.1)


def test_lists_that_are_not_of_tensors():
    x = torch.zeros(4, 8)
    for call in (lambda: nuts.nuts_norm([x, 1.0]), lambda: nuts.nuts_norm([x.to_sparse()]), lambda: nuts.Moments([x], states=([3], [x.clone()])),
                 lambda: nuts.nuts_adamw(nuts.Moments([x]), ["x"], step=1, lr=0.1)):
        with pytest.raises((TypeError, AttributeError, ValueError)):
            call()


def test_tables_are_read_from_lists():
    from array import array
    from paper_1910_11141_amd import learning as G
    x = [torch.zeros(4, 8), torch.zeros(5), None, torch.nn.Parameter(torch.zeros(2, 3))]
    table = array("q", [-7] * 20)
    assert G._read(x, None, table, 5, 1, 2, 4) == G._MOVED
    at = [t.data_ptr() if t is not None else 0 for t in x]
    assert table.tolist() == [-7, at[0], 32, -7, 0, -7, at[1], 5, -7, 0, -7, 0, 0, -7, -7, -7, at[3], 6, -7, 0]
    assert G._read(x, None, table, 5, 1, 2, 4) == 0
    assert G._read(x, [torch.zeros(4, 8), torch.zeros(5), torch.zeros(1), torch.zeros(6)], table, 5, 1) == G._OTHER_SHAPES
    assert G._read([x[0], x[1].half()], None, table, 5, 3, -1, 4) == G._SEVERAL_TYPES | G._MOVED and table[4::5].tolist()[:2] == [0, 3]
    assert G._read([x[0].t()], None, table, 5, 1) == G._GAPS
    assert G._read([torch.zeros(3, dtype=torch.int8)], None, table, 5, -1, -1, 0) == 0 and table[0] == -1
    assert G._read([], None, table, 5, 1) == 0
    for bad in ((None, None), ((x[0],), None), ([x[0]], [])):
        with pytest.raises(TypeError):
            G._read(*bad, table, 5, 1)


def test_numbers_that_the_library_refuses():
    x = torch.zeros(4, 8)
    for call in (lambda: nuts.nuts_penalties(x, repetition=0.0), lambda: nuts.nuts_penalties(x, frequency=NAN),
                 lambda: nuts.nuts_penalties(x, bias_ids=torch.zeros(4, 1025, dtype=torch.int64), bias_values=torch.zeros(4, 1025)),
                 lambda: nuts.nuts_penalties(x[:1].expand(4, 8)), lambda: nuts.nuts_norm([x], max_norm=0.0),
                 lambda: nuts.nuts_adamw(nuts.Moments([x]), [x.clone()], step=0, lr=0.1)):
        with pytest.raises(B.NutsError) as e:
            call()
        assert e.value.code == B.NUTS_E_INVALID_ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="what happens without a GPU")
def test_without_a_gpu_the_library_says_so():
    x, ids = torch.zeros(4, 8), torch.zeros(4, 3, dtype=torch.int64)
    for call in (lambda: nuts.nuts_penalties(x, ids), lambda: nuts.nuts_penalties(x, ids, out=x), lambda: nuts.nuts_penalties_grad(x, x, ids, want_bias=True),
                 lambda: nuts.nuts_norm([x]), lambda: nuts.nuts_adamw(nuts.Moments([x]), [x.clone()], step=1, lr=0.1),
                 lambda: nuts.nuts_adamw(nuts.Moments([x], bits=8), [x.clone()], step=1, lr=0.1), lambda: nuts.nuts_adamw_values(nuts.Moments([x], bits=8))):
        with pytest.raises(B.NutsError) as e:
            call()
        assert e.value.code == B.NUTS_E_DEVICE
    assert nuts.nuts_adamw(nuts.Moments([x]), [None], step=1, lr=0.1) is None


def test_names_are_the_packages():
    from paper_1910_11141_amd import learning
    for name in learning.__all__:
        assert getattr(nuts, name) is getattr(learning, name)
    code = ("import sys, paper_1910_11141_amd as n; n.NUTS_OK, n.Target; assert 'torch' not in sys.modules; n.nuts_adamw, n.Moments, n.nuts_penalties; "
            "assert 'nuts_adamw' in vars(n)")
    subprocess.run([sys.executable, "-c", code], check=True)


def test_random_bits_are_the_oracles():
    """The reference's Philox against the sampler's oracle, which is pinned by published vectors."""
    w = L.philox(torch.tensor([0, 0xffffffff]), torch.tensor([0, 0xffffffff]), torch.tensor([0, 0xffffffff]), torch.tensor([0, 0xffffffff]), 0)
    assert [int(x[0]) for x in w] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    w = L.philox(*[torch.tensor([0xffffffff])] * 4, 0xffffffffffffffff)
    assert [int(x[0]) for x in w] == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


@pytest.mark.skipif(torch.cuda.is_available(), reason="parameters on the CPU")
@pytest.mark.parametrize("bits", [32, 8])
def test_copies_of_moments_have_memory_of_their_own(bits, tmp_path):
    p = torch.nn.Parameter(torch.ones(300))
    mo = nuts.Moments([p, torch.zeros(5)], bits=bits, copies=[torch.zeros(300, dtype=torch.bfloat16), None])
    mo.v[0][:3] = 3
    torch.save(mo, tmp_path / "moments")
    model, twin = copy.deepcopy((p, mo))
    for other in (twin, torch.load(tmp_path / "moments", weights_only=False), copy.copy(mo)):
        addresses = other._now()[:]
        for i in range(2):
            tensors = (other.params[i], None, other.copies[i], other.m[i], other.v[i], other.m_scales[i], other.v_scales[i])
            assert [t.data_ptr() if t is not None else 0 for t in tensors] == list(addresses[8 * i:8 * i + 7])
            assert addresses[8 * i + 7] == (300, 5)[i]
        assert other.bits == bits and torch.equal(other.v[0], mo.v[0]) and torch.equal(other.params[0], p)
    assert twin.params[0] is model and twin.m[0].data_ptr() != mo.m[0].data_ptr()


def test_parameters_of_moments_stay_in_number():
    if torch.cuda.is_available():
        pytest.skip("parameters on the CPU")
    mo = nuts.Moments([torch.zeros(3)])
    assert all(isinstance(some, tuple) for some in (mo.params, mo.copies, mo.m, mo.v, mo.m_scales, mo.v_scales))


@pytest.mark.skipif(torch.cuda.is_available(), reason="parameters on the CPU")
@pytest.mark.parametrize("part", [lambda p: p[:2], lambda p: p.t(), lambda p: p.view(torch.int8)])
@pytest.mark.parametrize("what", ["parameter", "copy"])
def test_parameters_and_copies_that_are_another_part_of_their_memory(part, what):
    p, c = torch.zeros(4, 4), torch.zeros(4, 4, dtype=torch.bfloat16)
    mo = nuts.Moments([p, torch.zeros(3)], copies=[c, None], bits=8)
    x = p if what == "parameter" else c
    x.data = part(x.data)
    for call in (lambda: nuts.nuts_adamw(mo, [torch.zeros(p.shape), torch.zeros(3)], step=1, lr=0.1), lambda: nuts.nuts_adamw_values(mo)):
        with pytest.raises(ValueError, match="changed its size, type or device"):
            call()


@pytest.mark.parametrize("field", ["param", "grad", "copy", "m", "v", "m_scale", "v_scale"])
def test_addresses_that_no_device_has(field):
    lib, bad = B.lib(), table(B.nuts_adamw_tensor, tensor(), tensor(**{field: 1 << 48 | 4096}))
    refused(lib.nuts_adamw(adamw(state_bits=8), bad, 2, None, None, None), "address")
    if field not in ("m_scale", "v_scale"):
        refused(lib.nuts_adamw(adamw(), bad, 2, None, None, None), "address")
    if field != "grad":
        refused(lib.nuts_adamw_values(bad, 2, B.NUTS_F32), "address")
