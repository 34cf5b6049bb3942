"""Capped attention of chunk rows where the values are far from 1 and the scores
at the cap's ends: outputs are averages of the values, so they are finite and
accurate whatever the scores, while 2^32 times the sum of a row's |v| is inside
fp32 (1540 keys of 2^70: 2^116; 9005 keys: 2^118)."""
import numpy as np
import pytest
import torch

from tests import _cache_bounds as Z
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import run

pytestmark = pytest.mark.gpu


def _inputs(sh, ctx, chk, kind, exponent, seed=3):
    """q and keys along one direction, so that every score's size is far past
    the cap and its sign is the key's: all up, all down, down and then up, up
    and then down, or (mixed) random keys with scores on both sides."""
    nq, nkv, hd = sh.n_q_heads, sh.n_kv_heads, sh.head_dim
    g = torch.Generator().manual_seed(seed)
    cache = R.make_cache(np.add(ctx, chk), nkv, hd, seed=seed)
    T = int(np.sum(chk))
    qkv = torch.randn(T, (nq + 2 * nkv) * hd, generator=g)
    if kind != "mixed":
        way = torch.randint(0, 2, (hd,), generator=g).float() * 2 - 1
        qkv[:, :nq * hd] = (8 * way).repeat(nq)
        for i, n in enumerate(np.add(ctx, chk)):
            t = torch.arange(int(n))
            sign = {"up": t >= 0, "down": t < 0, "down_up": t >= n // 2, "up_down": t < n // 2}[kind].float() * 2 - 1
            cache.k[cache.bt[i][t // 16].long(), :, t % 16] = (8 * sign[:, None] * way).to(torch.bfloat16)[:, None]
    else:
        qkv[:, :nq * hd] *= 40
    cache.v = (cache.v.float() * 2.0 ** exponent).to(torch.bfloat16)   # exact: the exponents have room
    return cache, qkv.to(torch.bfloat16)


@pytest.mark.parametrize("kind", ["up", "down", "down_up", "up_down", "mixed"])
@pytest.mark.parametrize("cap", [20.0, 50.0, 64.0, 1000.0])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
def test_values_of_any_size(heads, cap, kind):
    sh, ctx, chk = R.shape(*heads), [1500, 0], [40, 130]
    for exponent in (0, 40, 70, -60):
        cache, qkv = _inputs(sh, ctx, chk, kind, exponent)
        got, ref, _, _ = run(sh, ctx, chk, cache=cache, qkv=qkv, softcap=cap, weights=True)
        m = Z.mass(sh, qkv, cache, ctx, chk, softcap=cap)
        # scores to the cap's ends: 8 fp32 half steps of the cap
        d = 2.0 ** -21 * cap
        assert np.isfinite(got[0]).all(), (exponent, np.isnan(got[0]).sum(), np.isinf(got[0]).sum())
        assert np.all(np.abs(got[0] - ref[0]) <= Z.bound(ref[0], m, 1540, d)), exponent
        assert np.all(np.abs(got[1] - ref[1]) <= d + 2.0 ** -22 * np.abs(ref[1]))
        assert np.allclose(got[2], ref[2], rtol=2 * d + 6e-5, atol=1e-6, equal_nan=True)


@pytest.mark.parametrize("kind", ["up", "down_up", "mixed"])
def test_values_of_any_size_where_keys_are_split(kind):
    sh, ctx, chk = R.shape(8, 2, 128), [9000], [5]
    for exponent in (0, 70):
        cache, qkv = _inputs(sh, ctx, chk, kind, exponent)
        got, ref, _, _ = run(sh, ctx, chk, cache=cache, qkv=qkv, softcap=50.0)
        m = Z.mass(sh, qkv, cache, ctx, chk, softcap=50.0)
        d = 2.0 ** -21 * 50
        assert np.all(np.abs(got[0] - ref[0]) <= Z.bound(ref[0], m, 9005, d)), exponent
        assert np.all(np.abs(got[1] - ref[1]) <= d + 2.0 ** -22 * np.abs(ref[1]))
