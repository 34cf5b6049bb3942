"""Capped scores at the cap's ends behind masks: what a row does not see, however
large, NaN or infinite, neither reaches it nor moves what its probabilities are
counted from."""
import numpy as np
import pytest
import torch

from tests import _cache_bounds as Z
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import run
from tests.test_gpu_cache_large_values import _inputs

pytestmark = pytest.mark.gpu

CTX, CHK = [700, 0, 90], [70, 200, 1]


def masks(kind):
    rng = np.random.default_rng(5)
    first = np.concatenate([c + np.arange(n) // 30 * 30 - 30 for c, n in zip(CTX, CHK)])
    first[[3, 100]] = 10 ** 9                                        # rows that see nothing
    return {"window": dict(window=45), "documents": dict(first=first), "prefix": dict(prefix=[740, 150, 0]),
            "all": dict(window=150, first=rng.integers(0, 60, sum(CHK)), prefix=[740, 150, 0])}[kind]


def compare(sh, cache, qkv, cap, kw, finite=True):
    got, ref, _, _ = run(sh, CTX, CHK, cache=cache, qkv=qkv, softcap=cap, weights=True, **kw)
    m, d = Z.mass(sh, qkv, cache, CTX, CHK, softcap=cap, **kw), 2.0 ** -21 * cap
    fine = np.isfinite(ref[0])
    assert fine.all() == finite and np.array_equal(fine, np.isfinite(got[0]))
    assert np.all((np.abs(got[0] - ref[0]) <= Z.bound(ref[0], m, 770, d))[fine])
    seen = np.isfinite(ref[1])
    assert np.array_equal(got[1][~seen], ref[1][~seen], equal_nan=True)
    assert np.all((np.abs(got[1] - ref[1]) <= d + 2.0 ** -22 * np.abs(ref[1]))[seen])
    assert np.allclose(got[2], ref[2], rtol=2 * d + 6e-5, atol=1e-6, equal_nan=True)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("mask", ["window", "documents", "prefix", "all"])
@pytest.mark.parametrize("kind", ["up", "down", "down_up", "up_down", "mixed"])
def test_scores_at_the_ends_behind_masks(heads, mask, kind):
    sh = R.shape(*heads)
    for cap, exponent in ((50.0, 0), (50.0, 60), (300.0, -60)):
        cache, qkv = _inputs(sh, CTX, CHK, kind, exponent)
        compare(sh, cache, qkv, cap, masks(mask))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf, 3e38])
@pytest.mark.parametrize("cap", [5.0, 50.0])
def test_hidden_keys_that_are_not_numbers(bad, cap):
    sh = R.shape(8, 2, 128)
    cache, qkv = _inputs(sh, CTX, CHK, "mixed", 0)
    # positions that no row behind a window of 45 sees
    for i, t in ((0, 10), (0, 600), (0, 655), (2, 3), (2, 40)):
        page, slot = cache.bt[i, t // 16].long(), t % 16
        cache.k[page, :, slot, 9] = bad
        cache.v[page, :, slot, 5] = bad
    compare(sh, cache, qkv, cap, dict(window=45))
    # and keys in the middle of a prompt, which some rows see: an infinite key scores +-cap, an infinite value stays one
    if np.isinf(bad):
        cache.v[cache.bt[1, 100 // 16].long(), :, 100 % 16, 5] = bad
        cache.k[cache.bt[1, 60 // 16].long(), :, 60 % 16, 9] = bad
        compare(sh, cache, qkv, cap, dict(window=45), finite=False)
