"""In place, 16 bytes in which nothing changes are left as they are.  NaNs that signal show it: a rounding to binary16 makes them quiet."""
import pytest
import torch

import categorical_ref as R
import paper_1910_11141_amd as nuts

pytestmark = pytest.mark.gpu

SIGNALS = 0x7c01   # (binary16)


def signalling(n, classes):
    return torch.full((n, classes), SIGNALS, dtype=torch.int16, device="cuda").view(torch.float16)


def changed(x, before):
    """[n, packs]: whether any of 8 numbers has other bits."""
    other = x.view(torch.int16) != before.view(torch.int16)
    return torch.nn.functional.pad(other, (0, -x.shape[1] % 8)).view(len(x), -1, 8).any(2)


def packs(n, classes, at):
    want = torch.zeros(n, -(-classes // 8), dtype=torch.bool, device="cuda")
    for row, v in at:
        want[row, v // 8] = True
    return want


@pytest.mark.parametrize("classes", [8, 21, 4096, 9003, 33000])
@pytest.mark.parametrize("own", [True, False])
def test_places_that_nothing_changes(classes, own):
    n = 90 if own else 3
    x = signalling(n, classes)
    out = torch.empty_like(x)
    nuts.nuts_penalties(x, torch.tensor([0], device="cuda"), repetition=1.5, out=out)
    assert bool(changed(out, x).all())    # (what is rounded is quiet)
    history = torch.tensor([2, classes - 1], device="cuda")
    at = [(row, int(v)) for row in range(n) for v in history]
    there = x.clone()
    nuts.nuts_penalties(there, history.expand(n, -1).contiguous() if own else history, repetition=1.5, out=there)
    assert torch.equal(changed(there, x), packs(n, classes, at))
    # a class that may not come, and one with a bias of its own
    mask = torch.ones(classes, dtype=torch.bool, device="cuda")
    mask[classes // 2] = False
    there = x.clone()
    nuts.nuts_penalties(there, allowed=R.pack_bits(mask), out=there)
    whole = classes // 8   # (fewer than 8 in the end are written as they were, beside a mask)
    assert torch.equal(changed(there, x)[:, :whole], packs(n, classes, [(row, classes // 2) for row in range(n)])[:, :whole])
    assert bool(there[:, 8 * whole:].isnan().all())
    there = x.clone()
    ids = (torch.arange(n, device="cuda")[:, None] * 7) % classes
    nuts.nuts_penalties(there, bias_ids=ids, bias_values=torch.ones(n, 1, device="cuda"), out=there)
    assert torch.equal(changed(there, x), packs(n, classes, [(row, int(v)) for row, v in enumerate(ids)]))
    # the gradient
    logits = torch.ones_like(x)
    out = nuts.nuts_penalties_grad(x, logits, history, repetition=1.5)[0]
    assert bool(changed(out, x).all())
    there = x.clone()
    nuts.nuts_penalties_grad(there, logits, history.expand(n, -1).contiguous() if own else history, repetition=1.5, out=there)
    assert torch.equal(changed(there, x), packs(n, classes, at))
