"""Paged cache: sizes whose indices would pass 31 bits are refused by the C entry points (nothing is launched)."""
import pytest

from test_paged_host import M, P, _attention, _cache, _lib

INT_MAX = 2 ** 31 - 1


def _weights(cache, hq, n, width=160):
    return _lib().skipffn_paged_weights(cache, hq, 0.1, n, P(1 << 44), hq * 8, P(1 << 43), None, P(1 << 42), width, None)


@pytest.mark.parametrize("dtype,path", [(0, 0), (0, 1), (1, 0)])
@pytest.mark.parametrize("group", [1, 7, 64])
def test_rows_of_one_sequence_past_31_bits(group, dtype, path):
    # rows: new tokens of a sequence x query heads of a kv head
    lib, most = _lib(), (INT_MAX - 4096) // group
    small = dict(heads_kv=1, head_dim=8, head_stride=8, row_stride=8, page_stride=128, dtype=dtype, path=path)
    size = lambda n, max_new: lib.skipffn_paged_attention_scratch_bytes(_cache(max_new=max_new, **small), group, n)
    assert size(most, most) > 0
    assert size(most, INT_MAX) > 0 and size(INT_MAX - 4096, most) > 0       # the smaller of the two counts
    if group > 1:
        big = _cache(max_new=INT_MAX, **small)
        for n in (most + 1, (1 << 31) // group, INT_MAX - 4096):
            assert size(n, INT_MAX) == 0
            assert _attention(big, hq=group, n=n, q=1 << 44, out=1 << 45, lse=1 << 43, scratch=1 << 46, ldq=group * 8, ldo=group * 8) == 2
            assert _weights(big, group, n) == 2


def _evict(cache, width=160, budget=16, into=None):
    return _lib().skipffn_paged_evict(cache, into, P(1 << 44), width, budget, 0, 0, P(1 << 45), P(1 << 43), P(1 << 46), None)


def test_columns_of_weights_rows_to_keep_and_sequences_past_31_bits():
    # loops that go past their last column, row or sequence by a CTA's step must not come round to negative ones
    for n in (INT_MAX, INT_MAX - 4096):
        assert _weights(_cache(), 32, 2, width=n) == 2
        assert _evict(_cache(), budget=n) == 2
        assert _evict(_cache(), width=n) == 2
        many = _cache(n_seq=n, table_width=1, table_stride=1)
        assert _lib().skipffn_paged_attention_scratch_bytes(many, 32, 2) == 0 and _attention(many) == 2
        assert _evict(many) == 2 and _lib().skipffn_paged_append(many, 2, P(300 * M), 1024, P(301 * M), 1024, None) == 2
