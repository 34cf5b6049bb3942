"""eb_op_rotary_kv_append with q/k norms into an 8-bit cache, and at positions
apart from the slots."""
import numpy as np
import pytest

from tests import _cache_ops as R
from tests.test_gpu_cache_rotary import check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,rdim", [((4, 2, 64), 0), ((4, 2, 64), 32), ((16, 2, 128), 0), ((16, 2, 128), 48)])
def test_norms_into_an_8_bit_cache(heads, rdim, layout):
    sh = R.shape(*heads, qk_norm=True)
    check(run(sh, [0, 40, 7], [20, 1, 3], rdim=rdim, layout=layout, fp8=True))
    pos = np.random.default_rng(2).integers(0, 2 ** 31 - 1, 24)
    check(run(sh, [0, 40, 7], [20, 1, 3], rdim=rdim, layout=layout, fp8=True, positions=pos, scaling="yarn", factor=4.0,
              length=4096))


@pytest.mark.parametrize("n", [1, 400])
def test_norms_of_narrow_and_wide_calls(n):
    sh = R.shape(32, 8, 128, qk_norm=True)
    check(run(sh, [5, 100], [n, 2], fp8=True))
    check(run(sh, [5, 100], [n, 2]))
