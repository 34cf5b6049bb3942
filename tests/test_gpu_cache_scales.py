"""eb_op_attention_mod at the ends of the scores' scale: products that leave
fp32's normal range on the way to the score are refused, the others are right.
(A scale that became 0 made NaN of the masked keys' scores of -inf.)"""
import numpy as np
import pytest

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import check, run

pytestmark = pytest.mark.gpu

FAKE = 0x10000   # refused before anything is read


@pytest.mark.parametrize("scale,k_scale,cap", [
    (1e-30, 1e-20, 0.0), (1e-38, 1.0, 0.0), (1e-45, 1.0, 0.0), (1e-36, 1.0, 1000.0), (1e-30, 1e-20, 1e-20),
    (1e30, 1e20, 0.0), (1e30, 1.0, 1e-9), (3e38, 2.0, 1000.0)])
def test_scales_that_leave_fp32_are_refused(scale, k_scale, cap):
    h = B.Handle(R.shape(8, 2, 64), 4, 64)
    kv = B.KvCache(FAKE, FAKE, 4, FAKE, 4, 1, k_scale, 1.0)
    for b in (B.HostBatch([3], [1]), B.HostBatch([3], [9])):
        assert B.lib().eb_op_attention_mod(h.h, FAKE, kv, b.c, B.score_mod(scale=scale, softcap=cap), FAKE, None, None, 0,
                                           FAKE, 1 << 30, None) == -2
        assert "fp32" in B.eb_last_error()


@pytest.mark.parametrize("scale,k_scale,cap", [(1e-20, 1e-15, 0.0), (1e-20, 1e-15, 30.0), (1e-15, 1e-15, 1e-15),
                                               (1e15, 1e-16, 0.0), (1e15, 1e-16, 30.0), (1e-11, 1e10, 0.0)])
@pytest.mark.parametrize("chk", [1, 40])
def test_scales_inside_fp32(scale, k_scale, cap, chk):
    sh = R.shape(4, 2, 64)
    cache = R.make_cache([100 + chk], 2, 64, True, 1)
    cache.scales = (float(np.float32(k_scale)), 0.25)
    got, ref, _, _ = run(sh, [100], [chk], cache=cache, scale=scale, softcap=cap, weights=True)
    check(got, ref)
