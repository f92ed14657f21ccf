"""The categorical operators' Python face: what loading it costs others, what calls are told apart, which shapes fit."""
import subprocess
import sys

import pytest
import torch

import paper_1910_11141_amd as nuts
from paper_1910_11141_amd import binding as B


def test_the_samplers_names_and_modules_need_no_categorical_ones():
    """Names of the binding and modules of the package are found without PyTorch, which the categorical operators import."""
    code = ("import sys, paper_1910_11141_amd as n; from paper_1910_11141_amd import build, workloads; n.NUTS_OK, n.Target, n.nuts_sample; "
            "assert not hasattr(n, 'no_such_name'); assert 'torch' not in sys.modules; "
            "n.nuts_lookup, n.Scores; assert 'torch' in sys.modules; assert 'nuts_lookup' in vars(n)")
    subprocess.run([sys.executable, "-c", code], check=True)


def test_all_names_of_the_operators_are_the_packages():
    from paper_1910_11141_amd import categorical
    for name in categorical.__all__:
        assert getattr(nuts, name) is getattr(categorical, name)
    with pytest.raises(AttributeError):
        nuts.no_such_name


def test_both_zeros_are_scales_of_their_own(monkeypatch):
    """0.0 == -0.0, but the rows' signs differ: what a call gives must not be what an earlier one with the other zero asked for."""
    import math
    from paper_1910_11141_amd import categorical
    seen = []
    monkeypatch.setattr(categorical, "_call", lambda entry, desc, *rest, **kw: seen.append(math.copysign(1.0, desc._obj.scale)))
    table, ids = torch.ones(7, 11), torch.zeros(3, dtype=torch.int64)
    for scale in (0.0, -0.0, 0.0):
        nuts.nuts_lookup(table, ids, scale=scale)
        nuts.nuts_lookup_grad(table[:3], ids, 7, scale=scale)
    assert seen == [1.0, 1.0, -1.0, -1.0, 1.0, 1.0]


def test_rows_must_lie_as_their_classes_do():
    """As many rows as classes are not enough: those of [3, 2] classes are not [2, 3] rows."""
    table, ids = torch.zeros(7, 11), torch.zeros(3, 2, dtype=torch.int64)
    for call in (lambda: nuts.nuts_lookup(table, ids, out=torch.zeros(2, 3, 11)), lambda: nuts.nuts_lookup(table, ids, out=torch.zeros(3, 22)),
                 lambda: nuts.nuts_lookup(table, ids, out=torch.zeros(66)), lambda: nuts.nuts_lookup(table, ids, out=torch.zeros(3, 11, 2).transpose(1, 2)),
                 lambda: nuts.nuts_lookup_grad(torch.zeros(2, 3, 11), ids, 7), lambda: nuts.nuts_lookup_grad(torch.zeros(3, 22), ids, 7),
                 lambda: nuts.nuts_lookup_grad(torch.zeros(66), ids, 7), lambda: nuts.nuts_lookup_grad(torch.zeros(()), ids, 7)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.skipif(torch.cuda.is_available(), reason="tensors without a GPU")
def test_rows_in_one_line_are_rows_too():
    table, ids = torch.zeros(7, 11), torch.zeros(3, 2, dtype=torch.int64)
    for call in (lambda: nuts.nuts_lookup(table, ids, out=torch.zeros(3, 2, 11)), lambda: nuts.nuts_lookup(table, ids, out=torch.zeros(6, 11)),
                 lambda: nuts.nuts_lookup(table, ids[0, 0], out=torch.zeros(11)), lambda: nuts.nuts_lookup_grad(torch.zeros(3, 2, 11), ids, 7),
                 lambda: nuts.nuts_lookup_grad(torch.zeros(6, 11), ids, 7), lambda: nuts.nuts_lookup_grad(torch.zeros(3, 2, 11), ids.view(-1), 7),
                 lambda: nuts.nuts_lookup_grad(torch.zeros(11), ids[0, 0], 7)):
        with pytest.raises(B.NutsError) as e:  # (of the shapes there is nothing to say)
            call()
        assert e.value.code == B.NUTS_E_DEVICE


def test_sizes_are_the_headers():
    """Each size that the header gives a range for is taken up to its end, and not beyond."""
    import ctypes as C
    import os
    import re
    from paper_1910_11141_amd import build
    with open(os.path.join(os.path.dirname(build.HERE), "include", "nuts.h")) as f:
        header = f.read()
    bytes_needed, checked = C.c_int64(), 0
    for struct, query, strides in ((B.nuts_lookup_desc, B.lib().nuts_lookup_grad_workspace, ("table_stride", "row_stride")),
                                   (B.nuts_logits_desc, B.lib().nuts_logprobs_workspace, ("row_stride",)),
                                   (B.nuts_score_desc, B.lib().nuts_score_workspace,
                                    ("x_stride", "weight_stride", "logits_stride", "grad_x_stride", "grad_weight_stride"))):
        text = re.search(r"typedef struct \{([^{}]*)\} " + struct.__name__ + ";", header).group(1)
        for name, low, high in re.findall(r"int\d+_t (\w+);\s*/\*[^*]*?(\d+) \.\. ([-0-9^ ]*[0-9]|NUTS_CAT_MAX_TOP)", text):
            low, high = int(low), eval(high.replace("^", "**"), {"NUTS_CAT_MAX_TOP": B.NUTS_CAT_MAX_TOP})
            for value, want in ((low - 1, B.NUTS_E_INVALID_ARG), (low, B.NUTS_OK), (high, B.NUTS_OK), (high + 1, B.NUTS_E_INVALID_ARG)):
                sizes = {k: 2 for k, t in struct._fields_ if t is C.c_int64 and k not in strides and k != "allowed_stride"}
                # (as long as a row: long strides have a limit of their own)
                stride = value + 1 if name == "dim" or (name == "n_classes" and struct is not B.nuts_lookup_desc) else 2
                desc = struct(**{**sizes, "scale": 1.0, **{k: max(stride, 2) for k in strides}, name: value})
                assert query(C.byref(desc), C.byref(bytes_needed)) == want, (struct.__name__, name, value)
            checked += 1
    assert checked == 3 + 3 + 3
