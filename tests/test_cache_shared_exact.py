"""Attention behind a common beginning is as exact as fcp_cache_attn is for the same sequences, however many rows a group brings together."""
import numpy as np
import pytest

import cache_ref as R
from paper_2602_21788_amd import binding as B
from test_cache_shared import Batch

one = lambda n: [(1 + i, 1) for i in range(n)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt, value", [("e4m3", 1.875), ("int8", 127)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq, hkv, groups", [(8, 2, [(1024, one(4))]), (8, 2, [(1024, one(12))]), (8, 2, [(1024, one(40))]), (4, 1, [(1024, [(9, 7)] * 2)]), (4, 1, [(1024, [(9, 7)] * 9)])])
def test_probabilities_keep_what_bf16_leaves(hq, hkv, groups, D, fmt, value):
    """Up to 32 rows of a sequence and KV head; 16, 48 and 160, 56 and 252 of a group.  All values are one number that bf16 holds, so O is that number whatever the probabilities are.  A key of
    every 64 has the greatest score and the others e = 0.5 + 0.49 * 2^-8 times its exponential, which bf16 rounds to 0.5.  By that alone sums would lose 0.49 * 2^-8 of 63/64 of their terms, and
    O, 32.5 / 32.62 of the number, lies nearer to the next lower bf16 number: 127 is 0.47 less, where these are 0.5 apart, and 1.875 0.0069, where they are 2^-7.  What the rounding leaves is
    at most 2^-8 of e; rounded in turn it is off by 2^-16 of e, and 1100 additions in 32 bits by 1100 * 2^-24: together less than 2^-13, a thirtieth of half a step of O."""
    import torch
    b = Batch(64, D, hq, hkv, groups, fmt, scale=float(-np.log(0.5 + 0.49 * 2.0 ** -8) / 64))
    b.ref.k_e[:], b.ref.v_e[:], b.ref.k[:] = 0, 0, R.encode(np.zeros(()), fmt)
    b.ref.k[:, :, 0, 0] = R.encode(np.full((), 64.0), fmt)
    b.ref.v[:] = R.encode(np.full((), float(value)), fmt)
    b.q[:] = 0
    b.q[:, :, 0] = 1
    b.cache = R.to_device(b.ref, torch, B)
    o, lse = b.run()
    assert (o == value).all(), np.unique(o)
