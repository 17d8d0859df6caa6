"""Attention over a paged cache on the GPU: what one row may depend on, values that are not numbers."""
import numpy as np
import pytest

from cache_util import Batch, within
from gpu_util import to_host

pytestmark = pytest.mark.gpu

PATHS = [("bf16", 0), ("bf16", 1), ("fp32", 0), ("fp32", 1)]
SHAPES = [
    # new, lens, hq, hk
    ((1, 2), (40, 3000), 8, 2),                              # a few rows, within one run and over many
    ((1, 1), (9, 700), 1, 1),
    ((12, 30), (50, 3000), 8, 2),                            # more rows
    ((300, 5), (310, 2000), 8, 2),                           # several tiles
]


def _check(x, out, lse, lost):
    """`lost` [tokens, heads]: rows that are no numbers; the others as the statement says."""
    r_out, r_lse, e_out, e_lse = x.want()
    got, got_lse = to_host(out), to_host(lse)
    assert np.isnan(got[lost]).all() and np.isnan(got_lse[lost]).all()
    keep = ~lost
    within(out[keep], r_out[keep], e_out[keep], "out")
    within(lse[keep], r_lse[keep], e_lse[keep], "lse")


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("new,lens,hq,hk", SHAPES)
def test_a_query_that_is_no_number_has_no_answer(new, lens, hq, hk, dtype, path):
    # every score of the row is NaN, so its result is, too: not the zeros of a row that sees nothing
    import torch
    x = Batch(31, new, lens, hq, hk, 64, 16, dtype, path=path)
    lost = np.zeros((x.cu[-1], hq), dtype=bool)
    for s in range(len(new)):
        lost[x.cu[s], 0] = lost[x.cu[s + 1] - 1, hq - 1] = True
    held = x.q.clone()
    x.q[torch.from_numpy(lost).cuda(), 3] = float("nan")
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    x.q = held
    _check(x, out, lse, lost)


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("new,lens,hq,hk", SHAPES)
def test_keys_that_are_no_numbers_reach_every_row_that_sees_them(new, lens, hq, hk, first, dtype, path):
    # the first block of the last sequence's keys alone, which is a piece of its own in a divided sequence, or most of them
    import torch
    x = Batch(32, new, lens, hq, hk, 64, 16, dtype, path=path)
    j = torch.arange(128 if first else lens[-1] * 3 // 4, device="cuda")
    x.k[x.d_table[-1].long()[j // 16], j % 16, hk - 1] = float("nan")
    lost = np.zeros((x.cu[-1], hq), dtype=bool)
    lost[x.cu[-2]:, hq - hq // hk:] = True
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    _check(x, out, lse, lost)
