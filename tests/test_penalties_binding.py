"""What the binding of penalties tells the library of a history: rows that are described as they lie, whatever their type becomes on the way."""
import pytest
import torch

import paper_1910_11141_amd as nuts
from paper_1910_11141_amd import categorical

LAYOUTS = {
    "dense": lambda h: h,
    "columns of a wider buffer": lambda h: torch.cat([h, h + 1, h + 2], 1)[:, :h.shape[1]],
    "later columns": lambda h: torch.cat([h + 1, h], 1)[:, h.shape[1]:],
    "every other row": lambda h: h.repeat_interleave(2, 0)[::2],
    "columns first": lambda h: h.t().contiguous().t(),
    "rows that overlap": lambda h: torch.as_strided(h, (4, 2), (1, 1)),
    "one row for all": lambda h: h[:1],
    "one row, expanded": lambda h: h[1].expand(4, -1),
    "one line": lambda h: h[2],
    "every other place": lambda h: h.repeat_interleave(2, 1)[:, ::2],
    "one place": lambda h: torch.cat([h, h], 1)[:, :1],
}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("ids,bias_ids", [(torch.int64, torch.int32), (torch.int32, torch.int64), (torch.int64, torch.int64), (torch.int32, torch.int32),
                                          (torch.int64, None), (torch.int32, None)])
def test_histories_are_described_as_they_lie(layout, ids, bias_ids, monkeypatch):
    history = LAYOUTS[layout](torch.arange(24).view(4, 6).to(ids))
    calls = []
    monkeypatch.setattr(categorical, "_call", lambda entry, desc, tensors, *more: calls.append((desc._obj, tensors)))
    kw = {}
    if bias_ids is not None:
        kw = dict(bias_ids=torch.cat([torch.arange(20).view(4, 5)] * 2, 1)[:, :5].to(bias_ids), bias_values=torch.ones(4, 5))
    nuts.nuts_penalties(torch.zeros(4, 50), history, **kw)
    if bias_ids is None:
        nuts.nuts_penalties_grad(torch.zeros(4, 50), torch.zeros(4, 50), history)
    for desc, tensors in calls:
        given = tensors[1] if tensors[1].dtype in categorical._ID_TYPES else tensors[2]   # (behind the logits, and the gradient's)
        assert desc.id_type == categorical._ID_TYPES[given.dtype] and desc.history_len == history.shape[-1]
        assert desc.history_stride == 0 or desc.history_stride >= desc.history_len
        read = torch.as_strided(given, (4, desc.history_len), (desc.history_stride, 1))
        assert torch.equal(read.long(), history.long().expand(4, -1))
        if bias_ids is not None:
            assert desc.n_bias == 5 and tensors[8].dtype == given.dtype and torch.equal(tensors[8].long(), torch.arange(20).view(4, 5)) and tensors[8].is_contiguous()
