"""eb_op_attention_mod with windows up to the largest int32: a window that
reaches past every key is none, in the outputs, the log-sum-exp and the weights
that the keys receive."""
import numpy as np
import pytest

from tests import _cache_ops as R
from tests.test_gpu_cache_attention import check, run

pytestmark = pytest.mark.gpu

WIDE = [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 1100, 2 ** 30]


@pytest.mark.parametrize("window", WIDE)
@pytest.mark.parametrize("heads,ctx,chk", [
    ((8, 2, 64), [0, 1000, 40, 700], [300, 70, 1, 3]),   # prompts, a chunk behind a context, decode rows
    ((8, 1, 128), [0], [1009]),                          # one prompt: its rows in parts
    ((8, 8, 64), [9000, 61], [3, 5]),                    # few rows over many keys: keys apart
])
def test_a_window_past_every_key_is_none(heads, ctx, chk, window):
    sh = R.shape(*heads)
    got, ref, _, _ = run(sh, ctx, chk, window=window, weights=True, softcap=20.0)
    check(got, ref)
    none = run(sh, ctx, chk, weights=True, softcap=20.0)[0]
    assert all(np.array_equal(a, b) for a, b in zip(got, none))


@pytest.mark.parametrize("window", WIDE)
def test_wide_windows_of_documents_and_a_prefix(window):
    sh, ctx, chk = R.shape(4, 2, 64), [200, 0], [90, 150]
    first = np.concatenate([200 + np.arange(90) // 30 * 30 - 100, np.arange(150) // 40 * 40])
    got, ref, _, _ = run(sh, ctx, chk, window=window, first=first, prefix=[250, 20], weights=True, weight_rows=60)
    check(got, ref)
