"""What AdamW's moments notice of tensors that have become others since they were given."""
import pytest
import torch

import paper_1910_11141_amd as nuts

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="parameters on the CPU")


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("which,other", [("parameters", torch.int32), ("bfloat16 parameters", torch.float16), ("copies", torch.float16), ("copies", torch.int16),
                                         ("the first copy", torch.float16), ("the last parameter", torch.int32)])
def test_types_that_change_where_the_numbers_lie(bits, n, which, other):
    """Address, number and shape are as they were, and all of a list's types change together, or one of them."""
    params = [torch.zeros(4, 4, dtype=torch.bfloat16 if which == "bfloat16 parameters" else torch.float32) for _ in range(n)]
    copies = [None] * (n // 2) + [torch.zeros(4, 4, dtype=torch.bfloat16) for _ in range(n - n // 2)]
    moments = nuts.Moments(params, copies=copies, bits=bits)
    given = [c for c in copies if c is not None]
    for t in {"copies": given, "the first copy": given[:1], "the last parameter": params[-1:]}.get(which, params):
        t.data = t.data.view(other)
    calls = [lambda: nuts.nuts_adamw(moments, [torch.zeros(4, 4)] * n, step=1, lr=0.1)]
    if bits == 8:
        calls.append(lambda: nuts.nuts_adamw_values(moments))
    for call in calls:
        with pytest.raises(ValueError, match="changed its size, type or device"):
            call()
