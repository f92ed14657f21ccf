"""The categorical operators refuse what they cannot do, on the host and before anything is written."""
import ctypes as C

import pytest
import torch

import categorical_ref as R
from paper_1910_11141_amd import binding as B
import paper_1910_11141_amd as nuts

P = C.c_void_p(4096)   # (never followed: a call that would has been refused)


def lookup(**kw):
    d = dict(dtype=0, id_type=0, n_ids=4, n_classes=5, dim=8, table_stride=8, row_stride=8, scale=1.0, accumulate=0, reserved=0)
    return C.byref(B.nuts_lookup_desc(**{**d, **kw}))


def logits(**kw):
    d = dict(dtype=0, id_type=0, n_rows=4, n_classes=5, row_stride=8, allowed_stride=0, scale=1.0, n_top=0, reserved=0)
    return C.byref(B.nuts_logits_desc(**{**d, **kw}))


def score(**kw):
    d = dict(dtype=0, id_type=0, n_rows=4, n_classes=5, dim=8, x_stride=8, weight_stride=8, logits_stride=8, grad_x_stride=8,
             grad_weight_stride=8, scale=1.0)
    return C.byref(B.nuts_score_desc(**{**d, **kw}))


def refused(rc, word=None):
    assert rc == B.NUTS_E_INVALID_ARG
    assert word is None or word in B.nuts_last_error(), B.nuts_last_error()


def test_struct_layouts():
    assert (C.sizeof(B.nuts_lookup_desc), C.sizeof(B.nuts_logits_desc), C.sizeof(B.nuts_score_desc)) == (64, 56, 80)


@pytest.mark.parametrize("bad,word", [
    (dict(dtype=1), "dtype"), (dict(dtype=4), "dtype"), (dict(id_type=2), "id_type"), (dict(n_ids=-1), "n_ids"), (dict(n_ids=2 ** 31), "n_ids"),
    (dict(n_classes=0), "n_classes"), (dict(n_classes=2 ** 31), "n_classes"), (dict(dim=0), "dim"), (dict(dim=2 ** 24 + 1), "dim"),
    (dict(table_stride=7), "stride"), (dict(row_stride=7), "stride"), (dict(table_stride=2 ** 61), "stride"), (dict(row_stride=2 ** 61), "stride"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(scale=1e300), "scale"), (dict(accumulate=2), "accumulate")])
def test_lookup_descriptors(bad, word):
    L, n = B.lib(), C.c_int64()
    refused(L.nuts_lookup(lookup(**bad), P, P, P), word)
    refused(L.nuts_lookup_grad(lookup(**bad), P, P, P, P, 1 << 40), word)
    refused(L.nuts_lookup_grad_workspace(lookup(**bad), C.byref(n)), word)


@pytest.mark.parametrize("bad,word", [
    (dict(dtype=1), "dtype"), (dict(id_type=-1), "id_type"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=2 ** 31 - 1), "n_rows"),
    (dict(n_classes=0), "n_classes"), (dict(n_classes=2 ** 31 - 1, row_stride=2 ** 31), "n_classes"), (dict(row_stride=4), "row_stride"),
    (dict(row_stride=2 ** 61), "row_stride"), (dict(n_classes=65, row_stride=65, allowed_stride=2), "allowed_stride"),
    (dict(allowed_stride=-1), "allowed_stride"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(scale=1e-60), "scale"), (dict(n_top=-1), "n_top"), (dict(n_top=65), "n_top")])
def test_logits_descriptors(bad, word):
    L, n = B.lib(), C.c_int64()
    refused(L.nuts_logprobs(logits(**bad), *[P] * 9, 1 << 40), word)
    refused(L.nuts_logprobs_workspace(logits(**bad), C.byref(n)), word)
    refused(L.nuts_logprobs_grad(logits(**bad), *[P] * 9, 1 << 31), word)


@pytest.mark.parametrize("bad,word", [
    (dict(dtype=1), "dtype"), (dict(dtype=3), "dtype"), (dict(id_type=7), "id_type"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=2 ** 20 + 1), "n_rows"),
    (dict(n_classes=0), "n_classes"), (dict(n_classes=2 ** 24 + 1, logits_stride=2 ** 25), "n_classes"), (dict(dim=0), "dim"),
    (dict(dim=2 ** 20 + 1), "dim"), (dict(x_stride=7), "stride"), (dict(weight_stride=7), "stride"), (dict(logits_stride=4), "stride"),
    (dict(grad_x_stride=7), "stride"), (dict(grad_weight_stride=7), "stride"), (dict(x_stride=2 ** 60), "stride"), (dict(scale=0.0), "scale"),
    (dict(scale=float("nan")), "scale")])
def test_score_descriptors(bad, word):
    L, n = B.lib(), C.c_int64()
    refused(L.nuts_score(score(**bad), *[P] * 8, 1 << 50), word)
    refused(L.nuts_score_grad(score(**bad), *[P] * 12, 1 << 50), word)
    refused(L.nuts_score_workspace(score(**bad), C.byref(n)), word)
    refused(L.nuts_score_grad_workspace(score(**bad), C.byref(n)), word)


def test_null_pointers_and_workspaces():
    L, n = B.lib(), C.c_int64()
    for call, args in ((L.nuts_lookup, (None, P, P, P)), (L.nuts_lookup_grad, (None, P, P, P, P, 0)), (L.nuts_logprobs, (None, *[P] * 9, 0)),
                       (L.nuts_logprobs_grad, (None, *[P] * 9, 0)), (L.nuts_score, (None, *[P] * 8, 0)), (L.nuts_score_grad, (None, *[P] * 12, 0)),
                       (L.nuts_lookup_grad_workspace, (None, C.byref(n))), (L.nuts_logprobs_workspace, (logits(), None)),
                       (L.nuts_score_workspace, (score(), None)), (L.nuts_score_grad_workspace, (score(), None)),
                       (L.nuts_lookup_grad_workspace, (lookup(), None))):
        refused(call(*args))
    refused(L.nuts_lookup(lookup(), None, P, P))
    refused(L.nuts_lookup(lookup(), P, None, P))
    refused(L.nuts_lookup(lookup(), P, P, None))
    refused(L.nuts_lookup_grad(lookup(), None, P, P, None, 0))
    refused(L.nuts_lookup_grad(lookup(), P, P, None, None, 0))
    many = lookup(n_ids=5000)
    assert L.nuts_lookup_grad_workspace(many, C.byref(n)) == B.NUTS_OK and n.value > 0
    refused(L.nuts_lookup_grad(many, P, P, P, P, n.value - 1), "workspace")
    refused(L.nuts_lookup_grad(many, P, P, P, None, n.value), "workspace")
    refused(L.nuts_lookup_grad(many, P, P, P, C.c_void_p(4097), n.value), "aligned")
    refused(L.nuts_logprobs(logits(), None, *[P] * 8, 0))
    long_rows = logits(n_classes=100000, row_stride=100000)
    assert L.nuts_logprobs_workspace(long_rows, C.byref(n)) == B.NUTS_OK and n.value > 0
    refused(L.nuts_logprobs(long_rows, *[P] * 9, n.value - 1), "workspace")
    refused(L.nuts_logprobs(long_rows, *[P] * 8, None, n.value), "workspace")
    refused(L.nuts_logprobs_grad(logits(), P, P, P, None, P, P, P, P, C.c_void_p(8192), 8))
    refused(L.nuts_logprobs_grad(logits(), P, P, P, P, None, P, P, P, C.c_void_p(8192), 8), "entropy")
    refused(L.nuts_logprobs_grad(logits(), P, P, P, P, P, P, P, P, C.c_void_p(8192), 4), "grad_stride")
    refused(L.nuts_logprobs_grad(logits(), P, P, P, P, P, P, P, P, P, 8), "overlap")
    refused(L.nuts_score(score(), None, *[P] * 7, 1 << 40))
    refused(L.nuts_score(score(), C.c_void_p(4100), *[P] * 7, 1 << 40), "16 bytes")
    assert L.nuts_score_workspace(score(), C.byref(n)) == B.NUTS_OK and n.value > 0
    refused(L.nuts_score(score(), *[P] * 8, n.value - 1), "workspace")
    refused(L.nuts_score_grad(score(), P, P, P, P, None, *[P] * 7, 1 << 40))
    refused(L.nuts_score_grad(score(), P, P, P, P, P, None, P, P, P, P, P, P, 1 << 40), "entropy")
    assert L.nuts_score_grad_workspace(score(), C.byref(n)) == B.NUTS_OK and n.value > 0
    refused(L.nuts_score_grad(score(), *[P] * 12, n.value - 1), "workspace")


def test_nothing_to_do_is_no_error():
    L, n = B.lib(), C.c_int64()
    for query, desc in ((L.nuts_lookup_grad_workspace, lookup(n_ids=0)), (L.nuts_logprobs_workspace, logits(n_rows=0)),
                        (L.nuts_score_workspace, score(n_rows=0)), (L.nuts_score_grad_workspace, score(n_rows=0))):
        assert query(desc, C.byref(n)) == B.NUTS_OK and n.value >= 0
    assert L.nuts_lookup(lookup(n_ids=0), None, None, None) == B.NUTS_OK
    assert L.nuts_logprobs(logits(n_rows=0), *[None] * 9, 0) == B.NUTS_OK
    assert L.nuts_logprobs_grad(logits(n_rows=0), *[None] * 9, 8) == B.NUTS_OK
    assert L.nuts_score(score(n_rows=0), *[None] * 8, 0) == B.NUTS_OK
    assert L.nuts_score_grad(score(), P, P, P, P, P, P, P, P, P, None, None, None, 0) == B.NUTS_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="what happens without a GPU")
def test_without_a_gpu_the_library_says_so():
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: nuts.nuts_lookup(x, ids), lambda: nuts.nuts_lookup_grad(x, ids, 5), lambda: nuts.nuts_logprobs(x, ids, n_top=2),
                 lambda: nuts.nuts_logprobs_grad(x, ids, torch.zeros(4)), lambda: nuts.nuts_score(x, x, ids),
                 lambda: nuts.nuts_score_grad(x, x, ids, torch.zeros(4))):
        with pytest.raises(B.NutsError) as e:
            call()
        assert e.value.code == B.NUTS_E_DEVICE


def test_tensors_that_do_not_fit():
    x, ids, f = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for call in (lambda: nuts.nuts_lookup(x.double(), ids), lambda: nuts.nuts_lookup(x.t(), ids), lambda: nuts.nuts_lookup(x[0], ids),
                 lambda: nuts.nuts_lookup(x, ids.float()), lambda: nuts.nuts_lookup(x, ids, out=torch.zeros(4, 7)),
                 lambda: nuts.nuts_lookup(x, ids, out=torch.zeros(4, 8).half()), lambda: nuts.nuts_lookup_grad(x, ids[:3], 5),
                 lambda: nuts.nuts_lookup_grad(x, ids, 5, accumulate=True), lambda: nuts.nuts_lookup_grad(x, ids, 5, out=torch.zeros(4, 8)),
                 lambda: nuts.nuts_logprobs(x, ids[:3]), lambda: nuts.nuts_logprobs(x, ids, allowed=torch.zeros(2, dtype=torch.int32)),
                 lambda: nuts.nuts_logprobs(x, ids, allowed=torch.zeros(3, 1, dtype=torch.int32)),
                 lambda: nuts.nuts_logprobs(x, ids, allowed=torch.zeros(4, 8, dtype=torch.bool)),
                 lambda: nuts.nuts_logprobs_grad(x, ids, f[:3]), lambda: nuts.nuts_logprobs_grad(x, ids, f, grad_logprob=f.double()),
                 lambda: nuts.nuts_logprobs_grad(x, ids, f, out=torch.zeros(4, 9)), lambda: nuts.nuts_score(x.half(), x.half(), ids),
                 lambda: nuts.nuts_score(x, x[:, :7], ids), lambda: nuts.nuts_score(x, x.bfloat16(), ids),
                 lambda: nuts.nuts_score_grad(x, x, ids, f, logits=torch.zeros(4, 5))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.NutsError):
        nuts.nuts_logprobs(x, ids, n_top=65)
    with pytest.raises(B.NutsError):
        nuts.nuts_logprobs(x, ids, scale=0.0)


def test_masks_are_packed_as_the_header_says():
    mask = torch.zeros(2, 70, dtype=torch.bool)
    mask[0, 0] = mask[0, 31] = mask[1, 32] = mask[1, 69] = True
    words = R.pack_bits(mask)
    assert words.tolist() == [[1 - 2 ** 31, 0, 0], [0, 1, 32]]
    assert torch.equal(R.bits(words, 70), mask)
