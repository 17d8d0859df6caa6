"""Paged cache and rotary positions: argument checks of the C entry points (nothing is launched)."""
import ctypes

import pytest

P = ctypes.c_void_p
M = 1 << 20


def _lib():
    import paper_2503_21817_b200 as sk
    return sk.load_library()


def _cache(**kw):
    from paper_2503_21817_b200.cache import _PagedCache
    f = dict(heads_kv=8, head_dim=128, dtype=0, path=0, page_size=16, n_seq=2, table_width=10, max_new=1, n_pages=100,
             k_pages=64 * M, v_pages=128 * M, page_stride=16 * 1024, row_stride=1024, head_stride=128, page_table=200 * M, table_stride=10,
             cu_new=201 * M, lens=202 * M, status=203 * M)
    f.update(kw)
    return ctypes.byref(_PagedCache(**f))


def _attention(cache, hq=32, scale=0.1, n=2, q=300 * M, ldq=4096, out=301 * M, ldo=4096, lse=302 * M, scratch=400 * M, nbytes=1 << 40):
    return _lib().skipffn_paged_attention(cache, hq, scale, n, P(q), ldq, P(out), ldo, P(lse), P(scratch), nbytes, None)


@pytest.mark.parametrize("status,bad", [
    (1, dict(heads_kv=0)), (1, dict(head_dim=0)), (2, dict(head_dim=12)), (2, dict(head_dim=136)), (1, dict(dtype=2)), (1, dict(path=2)),
    (1, dict(page_size=0)), (2, dict(page_size=12)), (1, dict(n_pages=-1)), (2, dict(n_pages=1 << 31)), (1, dict(n_seq=-1)),
    (1, dict(table_width=-1)), (1, dict(max_new=-1)), (1, dict(k_pages=None)), (1, dict(v_pages=128 * M + 8)), (1, dict(k_pages=64 * M + 2)),
    (1, dict(row_stride=1020)), (1, dict(row_stride=512)), (1, dict(head_stride=64)), (1, dict(page_stride=8 * 1024)), (1, dict(page_stride=-1)),
    (1, dict(page_table=None)), (1, dict(page_table=200 * M + 2)), (1, dict(table_stride=9)), (1, dict(cu_new=None)), (1, dict(lens=None)),
    (1, dict(lens=202 * M + 1)), (1, dict(status=None)), (1, dict(v_pages=64 * M)), (1, dict(v_pages=64 * M + 4096)),
    (2, dict(heads_kv=65536, head_stride=128, row_stride=128 * 65536, page_stride=128 * 65536 * 16))])
def test_caches_refused(status, bad):
    lib, c = _lib(), _cache(**bad)
    assert _attention(c) == status
    assert lib.skipffn_paged_append(c, 2, P(300 * M), 1024, P(301 * M), 1024, None) == status
    assert lib.skipffn_paged_weights(c, 32, 0.1, 2, P(300 * M), 4096, P(302 * M), None, P(303 * M), 160, None) == status
    assert lib.skipffn_paged_evict(c, None, P(300 * M), 160, 16, 0, 0, P(301 * M), P(302 * M), P(303 * M), None) == status
    assert lib.skipffn_paged_attention_scratch_bytes(c, 32, 2) == 0


def test_layouts_that_no_row_shares():
    # interleaved at the level of pages, rows, heads; heads outside rows: all are laid out, the scratch has a size
    size = lambda **kw: _lib().skipffn_paged_attention_scratch_bytes(_cache(**kw), 32, 2)
    assert size() > 0
    assert size(page_stride=32 * 1024, v_pages=64 * M + 32 * 1024) > 0
    assert size(row_stride=2048, page_stride=32 * 1024, v_pages=64 * M + 2048) > 0
    assert size(head_stride=256, row_stride=2048, page_stride=32 * 1024, v_pages=64 * M + 256) > 0
    assert size(head_stride=16 * 128, row_stride=128) > 0
    assert size(row_stride=2048, page_stride=32 * 1024, v_pages=64 * M + 1024) == 0      # half a row of heads further
    assert size(row_stride=2048, page_stride=33 * 1024, v_pages=64 * M + 2048) == 0      # pages that drift over the rows
    # one page, one row a page, one head: the strides of those levels do not count
    assert size(n_pages=1, page_stride=0) > 0 and size(heads_kv=1, head_stride=0) > 0


def test_attention_arguments_refused():
    lib, c = _lib(), _cache()
    assert _attention(None) == 1
    for kw in (dict(hq=0), dict(hq=12), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(n=-1),
               dict(q=None), dict(out=None), dict(lse=None), dict(scratch=None), dict(q=300 * M + 8), dict(ldq=4092), dict(ldq=4088), dict(ldq=-8),
               dict(ldo=1 << 40), dict(lse=302 * M + 2), dict(scratch=400 * M + 8), dict(out=300 * M), dict(out=300 * M + 4096), dict(lse=300 * M + 4),
               dict(lse=301 * M), dict(scratch=299 * M), dict(out=64 * M), dict(lse=128 * M + 64), dict(scratch=60 * M), dict(out=200 * M),
               dict(lse=201 * M), dict(scratch=202 * M), dict(out=203 * M)):
        assert _attention(c, **kw) == 1, kw
    assert _attention(c, hq=8 * 65, ldq=1 << 17, ldo=1 << 17) == 2
    assert _attention(c, nbytes=lib.skipffn_paged_attention_scratch_bytes(c, 32, 2) - 1) == 3
    assert lib.skipffn_paged_attention_scratch_bytes(c, 12, 2) == lib.skipffn_paged_attention_scratch_bytes(c, 32, -1) == 0
    assert _attention(c, n=0, q=None, out=None, lse=None) == 0                           # nothing to do
    assert lib.skipffn_paged_poll(None, None, None) == 1


def test_weights_and_append_arguments_refused():
    lib, c = _lib(), _cache()
    w = lambda hq=32, scale=0.1, n=2, q=300 * M, ldq=4096, lse=302 * M, prior=None, out=303 * M, width=160: lib.skipffn_paged_weights(
        c, hq, scale, n, P(q), ldq, P(lse), P(prior), P(out), width, None)
    for kw in (dict(hq=12), dict(scale=0.0), dict(n=-1), dict(q=None), dict(lse=None), dict(out=None), dict(width=-1), dict(ldq=4088),
               dict(out=303 * M + 2), dict(prior=305 * M + 1), dict(out=300 * M), dict(out=302 * M), dict(out=64 * M), dict(out=128 * M + 4),
               dict(prior=303 * M + 4), dict(out=202 * M)):
        assert w(**kw) == 1, kw
    assert w(width=0) == 0
    a = lambda n=2, k=300 * M, ldk=1024, v=301 * M, ldv=1024: lib.skipffn_paged_append(c, n, P(k), ldk, P(v), ldv, None)
    for kw in (dict(n=-1), dict(k=None), dict(v=None), dict(ldk=1016), dict(ldv=1020), dict(k=300 * M + 8), dict(k=64 * M), dict(v=128 * M + 1024)):
        assert a(**kw) == 1, kw
    assert a(n=0, k=None, v=None) == 0


def test_evict_arguments_refused():
    lib, c = _lib(), _cache()
    e = lambda into=None, w=300 * M, width=160, budget=16, sinks=2, recent=4, kept=301 * M, lens=302 * M, out=303 * M: lib.skipffn_paged_evict(
        c, into, P(w), width, budget, sinks, recent, P(kept), P(lens), P(out), None)
    other = dict(k_pages=500 * M, v_pages=600 * M)
    for kw in (dict(w=None), dict(width=-1), dict(budget=0), dict(budget=-1), dict(sinks=-1), dict(recent=-1), dict(sinks=13), dict(kept=None),
               dict(lens=None), dict(out=None), dict(kept=301 * M + 2), dict(kept=300 * M), dict(out=300 * M + 4), dict(lens=301 * M),
               dict(out=301 * M + 64), dict(kept=64 * M), dict(out=128 * M), dict(lens=202 * M), dict(into=_cache(**other, dtype=1)),
               dict(into=_cache(**other, heads_kv=4)), dict(into=_cache(**other, head_dim=64)), dict(into=_cache(**other, n_seq=1)),
               dict(into=_cache(**other, n_pages=-1)), dict(into=_cache(**other), kept=500 * M), dict(into=_cache(page_size=32, page_stride=32 * 1024)),
               dict(into=_cache(table_stride=16))):
        assert e(**kw) == 1, kw
    assert lib.skipffn_paged_evict(_cache(n_seq=0, cu_new=None, lens=None), None, None, 0, 16, 0, 0, None, None, None, None) == 0


def _rotary(freq=None, axis=None, hq=32, hk=8, d=128, rot=128, inter=0, axes=1, eps=1e-6):
    from paper_2503_21817_b200.cache import _RotaryConfig
    n = max(rot // 2, 1)
    f = (ctypes.c_double * n)(*([1.0] * n if freq is None else freq))
    x = None if axis is None else (ctypes.c_int32 * n)(*axis)
    cfg, h = _RotaryConfig(hq, hk, d, rot, inter, axes, None if freq == () else f, x, eps), P()
    return _lib().skipffn_rotary_create(ctypes.byref(h), ctypes.byref(cfg)), h


@pytest.mark.parametrize("status,bad", [
    (1, dict(hq=0)), (1, dict(hk=0)), (1, dict(d=0)), (2, dict(d=12, rot=8)), (2, dict(d=264, rot=8)), (2, dict(rot=12)), (1, dict(rot=136)),
    (1, dict(rot=-8)), (1, dict(inter=2)), (1, dict(axes=0)), (2, dict(axes=5)), (1, dict(eps=-1.0)), (1, dict(eps=float("nan"))),
    (1, dict(eps=float("inf"))), (1, dict(freq=())), (1, dict(freq=[float("nan")] * 64)), (1, dict(axis=[1] * 64)), (1, dict(axis=[-1] * 64)),
    (2, dict(hq=65536))])
def test_rotary_configurations_refused(status, bad):
    st, h = _rotary(**bad)
    assert st == status and not h.value


def test_rotary_arguments_refused():
    lib = _lib()
    st, h = _rotary(axes=2, axis=[0, 1] * 32)
    assert st == 0 and lib.skipffn_rotary_scratch_bytes(h) > 0 and lib.skipffn_rotary_scratch_bytes(None) == 0
    base = dict(q=300 * M, k=301 * M, pos=302 * M, gq=None, gk=None, oq=303 * M, ok=304 * M)
    f = lambda dt=0, n=5, ldq=4096, ldk=1024, ldp=5, ldoq=4096, ldok=1024, **kw: (lambda a: lib.skipffn_rotary_forward(
        h, dt, n, P(a["q"]), ldq, P(a["k"]), ldk, P(a["pos"]), ldp, P(a["gq"]), P(a["gk"]), P(a["oq"]), ldoq, P(a["ok"]), ldok, None))({**base, **kw})
    g = dict(gq=310 * M, gk=311 * M)
    for kw in (dict(dt=2), dict(n=-1), dict(n=1 << 31), dict(ldq=4088), dict(ldk=1020), dict(ldp=4), dict(ldoq=4088), dict(ldok=-8), dict(q=None),
               dict(k=None), dict(pos=None), dict(oq=None), dict(ok=None), dict(gq=310 * M), dict(gk=310 * M), dict(gq=310 * M + 8, gk=311 * M),
               dict(q=300 * M + 8), dict(oq=300 * M + 4096), dict(oq=301 * M), dict(ok=300 * M), dict(ok=303 * M), dict(oq=302 * M), dict(ok=301 * M + 16),
               dict(g, oq=310 * M), dict(g, ok=311 * M), dict(oq=300 * M, ldoq=8192)):
        assert f(**kw) == 1, kw
    assert lib.skipffn_rotary_forward(None, 0, 5, *[P(M), 4096] * 2, P(M), 5, None, None, *[P(M), 4096] * 2, None) == 1
    assert f(n=0, q=None, k=None, oq=None, ok=None, pos=None) == 0
    bb = dict(base, dyq=320 * M, dyk=321 * M, dq=330 * M, dk=331 * M, dgq=340 * M, dgk=341 * M, sc=350 * M, **g)
    b = lambda n=5, nb=1 << 30, dw=0, **kw: (lambda a: lib.skipffn_rotary_backward(
        h, 0, n, P(a["dyq"]), 4096, P(a["dyk"]), 1024, P(a["q"]), 4096, P(a["k"]), 1024, P(a["pos"]), n, P(a["gq"]), P(a["gk"]), P(a["dq"]), 4096,
        P(a["dk"]), 1024, P(a["dgq"]), P(a["dgk"]), dw, P(a["sc"]), nb, None))({**bb, **kw})
    arrays = ("dyq", "dyk", "q", "k", "pos", "gq", "gk")
    for o in ("dq", "dk", "dgq", "dgk", "sc"):
        for i in arrays:
            if (o, i) not in (("dq", "dyq"), ("dq", "q"), ("dk", "dyk"), ("dk", "k")):
                assert b(**{o: bb[i]}) == 1, (o, i)
        for i in ("dq", "dk", "dgq", "dgk", "sc"):
            if i != o:
                assert b(**{o: bb[i]}) == 1, (o, i)
    assert b(sc=None) == b(dw=2) == b(dyq=None) == b(dk=None) == b(sc=350 * M + 8) == b(dgq=340 * M + 1) == b(dw=1, dgk=341 * M + 2) == 1
    assert b(nb=lib.skipffn_rotary_scratch_bytes(h) - 1) == 3
    c = _cache()
    ap = lambda cache=c, hh=h, n=2, q=300 * M, k=301 * M, v=305 * M, oq=303 * M, ldv=1024, pos=302 * M: lib.skipffn_rotary_append(
        hh, cache, n, P(q), 4096, P(k), 1024, P(v), ldv, P(pos), 5, None, None, P(oq), 4096, None)
    for kw in (dict(cache=None), dict(hh=None), dict(cache=_cache(heads_kv=4)), dict(cache=_cache(head_dim=64)), dict(v=None), dict(ldv=1016),
               dict(oq=301 * M), dict(oq=305 * M), dict(oq=64 * M), dict(k=64 * M), dict(v=128 * M), dict(q=64 * M), dict(pos=64 * M), dict(oq=201 * M)):
        assert ap(**kw) == 1, kw
    lib.skipffn_rotary_destroy(h)
    lib.skipffn_rotary_destroy(None)


def test_python_refusals_without_a_device():
    import torch
    import paper_2503_21817_b200 as sk
    z = torch.zeros(4, 16, 2, 64)
    i = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        sk.PagedCache(z, z.clone(), i, i[0, :3], i[0, :2], 1)    # no CPU path
    with pytest.raises(ValueError):
        sk.RotaryQK(8, 2, 64, sections=[16, 8])
    with pytest.raises(ValueError):
        sk.RotaryQK(8, 2, 64, inv_freq=[1.0] * 31)
    with pytest.raises(sk.SkipFFNError):
        sk.RotaryQK(8, 2, 60)
    with pytest.raises(TypeError):
        sk.RotaryQK(8, 2, 64.5)
    rot = sk.RotaryQK(8, 2, 64)
    with pytest.raises(ValueError):
        rot.forward(torch.zeros(3, 8, 64), torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32))


def test_runs_cover_every_unit_once_and_none_is_empty():
    # the arithmetic of struct Runs (paged.cuh), in Python's integers
    for ctas in (1, 2, 7, 296):
        for units in (1, 2, 6, 8, 295, 296, 297, 1000, 3 * 10 ** 9):
            n = min(units, ctas)
            begin = [units * b // n if b < n else units for b in range(ctas + 1)]
            assert begin[0] == 0 and begin[n] == units and all(begin[b] < begin[b + 1] for b in range(n))
            for b in range(n):
                for u in (begin[b], begin[b + 1] - 1):
                    assert ((u + 1) * n - 1) // units == b
