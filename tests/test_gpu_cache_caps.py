"""eb_op_attention_mod with caps to 1000: a capped score keeps fp32's precision
whatever the cap.

Tolerances.  A capped score is off by a few fp32 half steps (2^-24) of its own
size, taken as 8: at most 2^-21 of the largest score.  The log-sum-exp is off by
that and two steps of its own size, a weight by twice that share of it and the
steps of its sum."""
import numpy as np
import pytest

from tests import _cache_bounds as Z
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import _qkv, check, run

pytestmark = pytest.mark.gpu

CAPS = [5.0, 50.0, 64.5, 100.0, 300.0, 1000.0]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
def test_ordinary_scores_under_any_cap(heads, cap, fp8):
    # scores to about 10 in size: the tolerance that all other masks and scores are tested with
    sh = R.shape(*heads)
    got, ref, _, _ = run(sh, [0, 700, 1100, 60, 90], [70, 33, 1, 1, 3], fp8=fp8, softcap=cap, weights=True)
    check(got, ref)
    slopes = [2.0 ** (-8.0 * (i + 1) / sh.n_q_heads) for i in range(sh.n_q_heads)]
    got, ref, _, _ = run(sh, [0, 300, 60], [70, 33, 1], fp8=fp8, softcap=cap, slopes=slopes, weights=True)
    check(got, ref)


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("scale", [0.5, 3.0, 40.0])
def test_scores_up_to_the_cap(cap, scale):
    sh, ctx, chk = R.shape(8, 2, 128), [300, 200, 500], [1, 60, 4]
    qkv = _qkv(65, sh, 2)
    cache = R.make_cache(np.add(ctx, chk), 2, 128, seed=1)
    got, ref, _, _ = run(sh, ctx, chk, cache=cache, qkv=qkv, softcap=cap, scale=scale, weights=True)
    # q has a deviation of 2: products to about 6 x 2 x sqrt(128) of the scale
    d = 2.0 ** -21 * min(cap, 140 * scale)
    assert np.all(np.abs(got[1] - ref[1]) <= d + 2.0 ** -22 * np.abs(ref[1])), np.abs(got[1] - ref[1]).max()
    assert np.allclose(got[2], ref[2], rtol=2 * d + 6e-5, atol=1e-6, equal_nan=True)
    m = Z.mass(sh, qkv, cache, ctx, chk, softcap=cap, scale=scale)
    assert np.all(np.abs(got[0] - ref[0]) <= Z.bound(ref[0], m, 504, d))
