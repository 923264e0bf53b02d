"""AdamwItems without a GPU: the tensors whose addresses it holds are its own to keep, whatever becomes of the lists they came in."""
import gc
import weakref

import pytest
import torch


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_outlive_the_lists_they_came_in(windq, monkeypatch, bits):
    monkeypatch.setattr(windq.binding, "_require_cuda", lambda *ts: None)
    state = torch.float32 if bits == 32 else torch.uint8
    lists = [[torch.zeros(300, dtype=t) for _ in range(3)] for t in (torch.float32, torch.bfloat16, state, state)]
    scales = [[torch.zeros(2) for _ in range(3)] for _ in range(2)] if bits == 8 else [None, None]
    copies = [torch.zeros(300, dtype=torch.bfloat16) for _ in range(3)]
    items = windq.AdamwItems(*lists, *scales, copies)
    held = [x for x in (*lists, *scales, copies) if x is not None]
    refs = [weakref.ref(t) for x in held for t in x]
    where = [t.data_ptr() for x in held for t in x]
    words = list(items._words)
    for x in held:
        x.clear()                                        # or refilled, or an entry replaced: the addresses stay these tensors'
    del x
    gc.collect()
    assert all(r() is not None and r().data_ptr() == at for r, at in zip(refs, where))
    assert list(items._words) == words and all(at in words for at in where)
    del items
    gc.collect()
    assert all(r() is None for r in refs)
