"""Penalties where a history and the ids of biases have different types, and rows of the history lie apart, against 64 bits."""
import pytest
import torch

import learning_ref as L
import paper_1910_11141_amd as nuts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,classes,length,room", [(2, 40, 5, 6), (7, 9001, 300, 777), (90, 32771, 40, 41)])
@pytest.mark.parametrize("ids,bias_ids", [(torch.int64, torch.int32), (torch.int32, torch.int64)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_said_before_in_a_growing_buffer(n, classes, length, room, ids, bias_ids, dtype):
    g = torch.Generator(device="cuda").manual_seed(n)
    said = torch.randint(-1, classes, (n, room), generator=g, device="cuda").to(ids)
    logits = torch.randn(n, classes, generator=g, device="cuda").to(dtype)
    kw = dict(repetition=1.5, frequency=0.5, presence=0.25, bias_ids=torch.randint(-2, classes + 2, (n, 3), generator=g, device="cuda").to(bias_ids),
              bias_values=torch.randn(n, 3, generator=g, device="cuda"))
    for history in (said[:, :length], said[:, room - length:], said[:1, :length], said[0, :length]):
        want, bound = L.penalties(logits, history, **kw)
        assert L.close(nuts.nuts_penalties(logits, history, **kw), want, bound)
