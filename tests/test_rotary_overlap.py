"""Rotary positions: results in place of an array that another kind of rows is read from are refused (nothing is launched)."""
import pytest

from test_paged_host import M, P, _cache, _lib, _rotary

Q, K, V, POS, OQ, OK = (M * i for i in (300, 301, 302, 303, 304, 305))
GQ, GK, DQ, DK, DGQ, DGK, SC = (M * i for i in (310, 311, 320, 321, 330, 331, 340))


@pytest.fixture
def handle():
    st, h = _rotary(hq=8, hk=8)
    assert st == 0
    yield h
    _lib().skipffn_rotary_destroy(h)


def test_forward(handle):
    f = lambda q, k, oq, ok: _lib().skipffn_rotary_forward(handle, 0, 5, P(q), 1024, P(k), 1024, P(POS), 5, None, None, P(oq), 1024, P(ok), 1024, None)
    # queries and keys may be one array, but then neither result may stand on it
    assert f(Q, Q, Q, OK) == 1
    assert f(Q, Q, OQ, Q) == 1
    assert f(Q, K, K, OK) == 1 and f(Q, K, OQ, Q) == 1


def test_append(handle):
    a = lambda q, k, v, oq: _lib().skipffn_rotary_append(handle, _cache(), 2, P(q), 1024, P(k), 1024, P(v), 1024, P(POS), 2, None, None, P(oq), 1024, None)
    assert a(Q, Q, V, Q) == 1 and a(Q, K, Q, Q) == 1 and a(Q, K, V, V) == 1


@pytest.mark.parametrize("norm", [False, True])
def test_backward(handle, norm):
    g = (GQ, GK, DGQ, DGK, SC) if norm else (None,) * 5
    b = lambda gq, gk, q, k, dq, dk: _lib().skipffn_rotary_backward(
        handle, 0, 5, P(gq), 1024, P(gk), 1024, P(q), 1024, P(k), 1024, P(POS), 5, P(g[0]), P(g[1]), P(dq), 1024, P(dk), 1024, P(g[2]), P(g[3]), 0,
        P(g[4]), 1 << 30, None)
    assert b(DQ, DQ, Q, K, DQ, OK) == 1                      # one upstream gradient for both
    assert b(DQ, DQ, Q, K, OQ, DQ) == 1
    assert b(DQ, DK, Q, Q, Q, OK) == 1                       # one input for both
    assert b(DQ, DK, Q, Q, OQ, Q) == 1
    assert b(DQ, Q, Q, K, Q, OK) == 1                        # the keys' upstream gradient in the queries' input
    assert b(K, DK, Q, K, OQ, K) == 1                        # and the other way round
