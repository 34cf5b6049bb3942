"""Request lengths past 32 bits are refused where a batch is made: numpy cuts an
int64 array off without a word."""
import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B


@pytest.mark.parametrize("bad", [np.array([5, 2 ** 32 + 3]), np.array([2 ** 31], np.uint32), np.array([-2 ** 31 - 1]),
                                 [2 ** 32 + 3, 1], torch.tensor([2 ** 40])])
def test_lengths_past_32_bits(bad):
    ones = [1] * len(bad)
    for pair in ((bad, ones), (ones, bad)):
        with pytest.raises((ValueError, OverflowError)):
            B.HostBatch(*pair)


@pytest.mark.parametrize("kind", [list, np.array, lambda a: np.array(a, np.int32), lambda a: np.array(a, np.uint8),
                                  torch.tensor, lambda a: np.array(a, np.uint64)])
def test_lengths_of_any_kind(kind):
    b = B.HostBatch(kind([5, 0, 7]), kind([1, 9, 2]))
    assert b.ctx.tolist() == [5, 0, 7] and b.chk.dtype == np.int32 and (b.c.num_seqs, b.c.num_tokens) == (3, 12)
    assert B.HostBatch([], []).c.num_seqs == 0
    assert B.HostBatch([2 ** 31 - 1], [1]).ctx[0] == 2 ** 31 - 1
