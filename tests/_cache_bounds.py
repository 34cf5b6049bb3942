"""How far an output of eb_op_attention_mod may be from the 64-bit definition,
element by element."""
from __future__ import annotations

import numpy as np
import torch

from tests import _cache_ops as R


def mass(sh, qkv, cache, ctx, chk, **kw) -> np.ndarray:
    """sum p |v| of every output: the same attention over the values' sizes."""
    v = cache.v & 0x7F if cache.scales is not None else cache.v.abs()
    return R.attend_batch(sh, qkv, R.Cache(cache.k, v, cache.bt, cache.scales), ctx, chk, **kw)[0]


def bound(ref_out, m, keys, score_error=3e-5) -> np.ndarray:
    """Each probability enters the product with the values rounded to bf16 (half
    a step: 2^-8 of it), and the output is rounded to bf16 once more.  A score
    that is off by score_error moves a probability by that share of it, and
    their sum again; fp32 sums over `keys` terms move it by 2^-24 each at most,
    and the division by the sum by a few more."""
    half = float(torch.finfo(torch.bfloat16).eps) / 2
    inner = (half + 2 * score_error + (keys + 8) * 2.0 ** -24) * m
    return inner + half * (np.abs(ref_out) + inner)
