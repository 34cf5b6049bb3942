"""Integers past 32 bits given to the binding of the cache operators: the
library's arguments hold 32, and what is cut off would be another window,
budget or count without a word."""
import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests.test_cache_ops_sizes import _kv, h  # noqa: F401

WIDE = [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 40]


@pytest.mark.parametrize("n", WIDE)
def test_structs(n):
    for make in (lambda: B.score_mod(window=n), lambda: B.rotary(1e4, rotary_dim=n), lambda: B.rotary(1e4, original_len=n)):
        with pytest.raises(ValueError, match="32 bits"):
            make()


@pytest.mark.parametrize("n", WIDE)
def test_arguments(h, n):  # noqa: F811
    x, b, kv, w = torch.zeros(2, 512, dtype=torch.bfloat16), B.HostBatch([3, 5], [1, 1]), _kv(), torch.zeros(4, 2, 16)
    with pytest.raises(ValueError, match="32 bits"):
        B.eb_op_attention_mod(h, x, kv, b, kv_weights=w, weight_rows=n)
    for kw in (dict(sink=n), dict(recent=n)):
        with pytest.raises(ValueError, match="32 bits"):
            B.eb_op_kv_evict(h, kv, w, [20, 20], [16, 16], _kv(), **kw)
    for bad in ([n, 20], np.array([n, 20])):
        with pytest.raises(ValueError, match="32 bits"):
            B.eb_op_kv_evict(h, kv, w, bad, [16, 16], _kv())
        with pytest.raises(ValueError, match="32 bits"):
            B.score_mod(prefix_lens=bad)


@pytest.mark.parametrize("n", [0, 5, 2 ** 31 - 1, np.int64(7), np.int32(7)])
def test_what_fits(n):
    assert B.score_mod(window=n).window == n and B.rotary(1e4, original_len=n).original_len == n
