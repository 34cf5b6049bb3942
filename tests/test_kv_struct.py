"""A cache struct keeps the tensors it points to: made from a temporary (block
tables just moved to the GPU, say) it would otherwise name memory that the next
allocation may write."""
import gc
import weakref

import pytest
import torch

from paper_2606_00516_amd import binding as B


@pytest.mark.parametrize("fp8", [False, True])
def test_the_struct_keeps_its_tensors(monkeypatch, fp8):
    monkeypatch.setattr(B, "_ptr", lambda t: t.data_ptr())
    k = torch.zeros(3, 2, 16, 64, dtype=torch.uint8 if fp8 else torch.bfloat16)
    v, bt = torch.zeros_like(k), torch.zeros(1, 3, dtype=torch.int32)
    refs = [weakref.ref(t) for t in (k, v, bt)]
    at = [t.data_ptr() for t in (k, v, bt)]
    kv = B.kv_struct(k, v, bt, (0.5, 0.25) if fp8 else None)
    del k, v, bt
    gc.collect()
    assert all(r() is not None for r in refs)
    assert [kv.k_cache, kv.v_cache, kv.block_tables] == at
    del kv
    gc.collect()
    assert all(r() is None for r in refs)
