"""Appending to a paged cache on the GPU while the integer tensors are at fault: reported, and nothing overwritten."""
import pytest

from cache_util import Batch, normal

pytestmark = pytest.mark.gpu

FAULTS = {
    # name: (cu, lens, sequences left out, site)
    "end past the call's tokens": ((0, 3, 5, 15), None, (2,), 64),
    "end far past the call's tokens": ((0, 3, 5, 2 ** 31 - 1), None, (2,), 64),
    "more than the most new tokens": ((0, 0, 0, 9), None, (2,), 64),
    "negative offset": ((-2, 3, 5, 9), None, (0,), 64),
    "descending": ((0, 3, -7, 9), None, (1, 2), 64),
    "first offset past zero": ((2, 3, 5, 9), None, (), 64),
    "length past the table": (None, (25, 9, 12), (0,), 65),
    "length far past the table": (None, (20, 2 ** 31 - 1, 12), (1,), 65),
    "negative length": (None, (20, 9, -3), (2,), 65),
    "length past the table of a sequence without tokens": ((0, 3, 3, 7), (20, 10 ** 6, 12), (1,), 65),
}


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fault", FAULTS)
def test_a_sequence_at_fault_is_reported_and_its_rows_stay(fault, dtype, turned):
    import torch
    import paper_2503_21817_b200 as sk
    new, lens, hq, hk, d, page, n = (3, 2, 4), (20, 9, 12), 4, 2, 16, 8, 9
    x = Batch(21, new, lens, hq, hk, d, page, dtype)             # a table of three pages: 24 rows
    q, k, v = (normal(i, n, h, d, dtype=dtype) for i, h in ((1, hq), (2, hk), (3, hk)))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rot = sk.RotaryQK(hq, hk, d)
    want_q, want_k = rot.forward(q, k, pos) if turned else (q, k)
    bad_cu, bad_lens, out, site = FAULTS[fault]
    cu, lens = bad_cu or x.cu, bad_lens or lens
    x.d_cu.copy_(torch.tensor(cu, dtype=torch.int32)), x.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    expect = x.k.clone(), x.v.clone()
    for s in range(3):
        for t in range(cu[s], cu[s + 1]) if s not in out else ():
            j = lens[s] - cu[s + 1] + t
            at = int(x.table[s, j // page]), j % page
            expect[0][at], expect[1][at] = want_k[t], v[t]
    if turned:
        got = rot.append(x.cache, q, k, v, pos, out_q=torch.full_like(q, 7.0))
    else:
        x.cache.append(k, v)
    with pytest.raises(sk.SkipFFNError, match=f"site {site}"):
        x.cache.poll()
    x.cache.poll()                                               # reported once
    for a, b in zip((x.k, x.v), expect):
        assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))
    if turned:                                                   # queries do not depend on the cache
        for s in range(3):
            if s not in out:
                assert torch.equal(got[cu[s]:cu[s + 1]], want_q[cu[s]:cu[s + 1]])
