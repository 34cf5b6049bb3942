"""Requests that share prefix pages and keep account of their keys' weights: one
call takes each page once (a call with a page twice is refused by a handle that
validates), calls after one another add up."""
import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import _qkv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("chk", [1, 20])
def test_weights_of_shared_pages_over_two_calls(chk, monkeypatch):
    sh, ctx = R.shape(8, 2, 64), [130, 100]
    cache = R.make_cache([130 + chk, 100 + chk], 2, 64, seed=3)
    bt = cache.bt.clone()
    bt[1, :6] = bt[0, :6]                                   # 96 keys of prefix in the same pages
    shared = R.Cache(cache.k, cache.v, bt, None)
    qkv = _qkv(2 * chk, sh, 4)
    w0 = torch.rand(cache.k.shape[:3], generator=torch.Generator().manual_seed(5))
    d, w, x = shared.cuda(), w0.cuda(), qkv.cuda()
    h, want, outs = B.Handle(sh, 2, 2 * chk), w0, []
    for i in range(2):
        rows = slice(i * chk, (i + 1) * chk)
        one = R.Cache(shared.k, shared.v, bt[i:i + 1].contiguous(), None)
        ref = R.attend_batch(sh, qkv[rows], one, ctx[i:i + 1], [chk], weights=want)
        want = torch.from_numpy(ref[2])
        kv = B.kv_struct(d.k, d.v, d.bt[i:i + 1].contiguous())
        outs.append(B.eb_op_attention_mod(h, x[rows].contiguous(), kv, B.HostBatch(ctx[i:i + 1], [chk]), kv_weights=w))
        torch.cuda.synchronize()
        assert np.allclose(R.f64(w), ref[2], rtol=6e-5, atol=1e-6)
    # without weights nothing is written to the shared pages: one call may take both
    both = B.eb_op_attention_mod(h, x, B.kv_struct(d.k, d.v, d.bt), B.HostBatch(ctx, [chk, chk]))
    torch.cuda.synchronize()
    assert torch.equal(both, torch.cat(outs))
    monkeypatch.setenv("EB_DEBUG_VALIDATE", "1")
    checked = B.Handle(sh, 2, 2 * chk)
    with pytest.raises(B.EbError, match="twice"):
        B.eb_op_attention_mod(checked, x, B.kv_struct(d.k, d.v, d.bt), B.HostBatch(ctx, [chk, chk]), kv_weights=w)
