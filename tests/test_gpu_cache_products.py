"""The products of probabilities and values of eb_op_attention_mod, each output
against its own bound (tests/_cache_bounds.py) instead of one for all: over long
contexts outputs are small, and a bound by the largest value would let the loss
of a whole split of the keys pass.

That the bound does see such a loss is shown on the CPU, with mistakes planted
in the oracle's outputs."""
import numpy as np
import pytest
import torch

from tests import _cache_bounds as Z
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import _qkv, run

HEADS = [(4, 4, 64), (8, 1, 64), (8, 2, 128), (16, 2, 128)]


def compare(sh, ctx, chk, fp8=False, seed=1, **kw):
    cache, qkv = R.make_cache(np.add(ctx, chk), sh.n_kv_heads, sh.head_dim, fp8, seed), _qkv(int(np.sum(chk)), sh, seed + 1)
    got, ref, _, _ = run(sh, ctx, chk, fp8=fp8, cache=cache, qkv=qkv, **kw)
    if kw.get("slopes") is not None:
        kw["slopes"] = np.asarray(kw["slopes"], np.float32)
    m = Z.mass(sh, qkv, cache, ctx, chk, **kw)
    off, most = np.abs(got[0] - ref[0]), Z.bound(ref[0], m, int(np.add(ctx, chk).max()))
    assert np.all(off <= most), (float((off / most).max()), np.argwhere(off > most)[:4])


@pytest.mark.gpu
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kw", [dict(), dict(softcap=20.0), dict(slopes=0.05), dict(softcap=30.0, slopes=0.1)])
def test_long_contexts(heads, fp8, kw):
    sh, kw = R.shape(*heads), dict(kw)
    if "slopes" in kw:
        kw["slopes"] = [kw["slopes"] / (i + 1) for i in range(sh.n_q_heads)]
    # decode rows of one split to more than 64; chunks of few rows split, of many rows whole
    compare(sh, [40000, 9000, 2047, 2048, 500], [1, 1, 1, 1, 1], fp8, **kw)
    compare(sh, [9000, 2500, 700, 0], [5, 2, 40, 150], fp8, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
def test_masks(heads, fp8):
    sh, ctx, chk = R.shape(*heads), [5000, 3000, 200, 0], [1, 6, 90, 300]
    compare(sh, ctx, chk, fp8, window=700, softcap=25.0)
    first = np.concatenate([c + np.arange(n) // 40 * 40 - back for c, n, back in zip(ctx, chk, (4000, 2000, 100, 0))])
    compare(sh, ctx, chk, fp8, first=first)
    compare(sh, ctx, chk, fp8, prefix=[5001, 3006, 250, 290], scale=0.3)


def _long_row(seed=3):
    """One row of 4 heads over 9001 keys of 128, its probabilities and values."""
    sh = R.shape(4, 4, 128)
    cache, qkv = R.make_cache([9001], 4, 128, seed=seed), _qkv(1, sh, seed)
    q = R.f64(qkv)[:, :512].reshape(1, 4, 128)
    k, v = R.gather(cache.k, cache.bt[0], 9001), R.gather(cache.v, cache.bt[0], 9001)
    out, _, p = R.attend(q, k, v, R.visible(9000, 1), 9000, softcap=50.0)
    return out[0], p[0], v, Z.mass(sh, qkv, cache, [9000], [1], softcap=50.0).reshape(4, 128)


def test_the_bound_sees_a_lost_split():
    out, p, v, m = _long_row()
    most = Z.bound(out, m, 9001)
    for per in (512, 1024):
        for k0 in range(0, 9001, per):
            part = np.einsum("ht,thd->hd", p[:, k0:k0 + per], v[k0:k0 + per])
            assert (np.abs(part) > most).any(axis=1).all(), (per, k0)       # lost: in every head
            swapped = np.roll(part, 1, axis=0) - part                       # another head's share
            assert (np.abs(swapped) > most).any(axis=1).all(), (per, k0)


def test_the_bound_lets_the_roundings_pass():
    out, p, v, m = _long_row()
    half = torch.finfo(torch.bfloat16).eps / 2
    assert half == 2.0 ** -8
    rounded = torch.from_numpy(p).to(torch.bfloat16).double().numpy()
    o = torch.from_numpy(np.einsum("ht,thd->hd", rounded, v)).to(torch.bfloat16).double().numpy()
    assert np.all(np.abs(o - out) <= Z.bound(out, m, 9001))
