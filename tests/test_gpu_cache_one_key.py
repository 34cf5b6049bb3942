"""Rows of eb_op_attention_mod that see one key get its value, bit for bit: the
probability is 1 whatever the score.  And where a few keys count, an output is
no further off than its own rounding and theirs."""
import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import _qkv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(softcap=5.0), dict(softcap=30.0), dict(softcap=50.0), dict(softcap=300.0),
                                dict(slopes=True), dict(softcap=30.0, slopes=True)])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("scale", [0.0, 3.0])
def test_a_row_that_sees_one_key_gets_its_value(heads, kw, scale):
    sh, ctx, chk = R.shape(*heads), [700, 0, 90, 2000, 30], [70, 200, 1, 3, 17]
    nq, nkv, hd = heads
    kw, T = dict(kw), sum(chk)
    if kw.pop("slopes", None):
        kw["slopes"] = torch.tensor([0.1 * (i + 1) for i in range(nq)], device="cuda")
    cache, qkv = R.make_cache(np.add(ctx, chk), nkv, hd, seed=2), _qkv(T, sh, 3)
    want, row = torch.zeros(T, nq, hd, dtype=torch.bfloat16), 0
    for i, (c, n) in enumerate(zip(ctx, chk)):
        p = torch.arange(c, c + n)
        v = cache.v[cache.bt[i][p // 16].long(), :, p % 16]
        want[row:row + n] = v.repeat_interleave(nq // nkv, dim=1)
        row += n
    d, h = cache.cuda(), B.Handle(sh, len(ctx), T)
    kv, b = B.kv_struct(d.k, d.v, d.bt), B.HostBatch(ctx, chk)
    out = B.eb_op_attention_mod(h, qkv.cuda(), kv, b, B.score_mod(scale=scale, window=1, **kw))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().view(T, nq, hd), want)
    # the key of its own position by documents of one
    first = torch.cat([torch.arange(c, c + n) for c, n in zip(ctx, chk)]).to(torch.int32).cuda()
    out = B.eb_op_attention_mod(h, qkv.cuda(), kv, b, B.score_mod(scale=scale, first_key=first, **kw))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().view(T, nq, hd), want)


@pytest.mark.parametrize("cap", [20.0, 50.0, 1000.0])
@pytest.mark.parametrize("window", [2, 100, 0])
def test_the_mean_error_of_peaked_rows(cap, window):
    """Scores with a deviation of 8: one or two keys of a row count.  Over many
    outputs the mean square of the output's own rounding is (2^-8)^2 / 12 / ln 2
    of it or less (uniform steps over a binade), a root of 1.4e-3 to 1.7e-3; the
    probabilities' roundings may add a quarter of that, not the 2^-8 of the
    largest one (2.3e-3 in all)."""
    sh, ctx, chk = R.shape(8, 2, 128), [1500, 0], [60, 200]
    cache, qkv = R.make_cache(np.add(ctx, chk), 2, 128, seed=4), _qkv(260, sh, 5, scale=8.0)
    ref = R.attend_batch(sh, qkv, cache, ctx, chk, window, softcap=cap)[0]
    d = cache.cuda()
    out = B.eb_op_attention_mod(B.Handle(sh, 2, 260), qkv.cuda(), B.kv_struct(d.k, d.v, d.bt), B.HostBatch(ctx, chk),
                                B.score_mod(softcap=cap, window=window))
    torch.cuda.synchronize()
    off = np.sqrt(((R.f64(out) - ref) ** 2).sum() / (ref ** 2).sum())
    assert off <= 2.1e-3, off
