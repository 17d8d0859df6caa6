"""Packed attention and layer normalisation: argument checks of the C entry points (nothing is launched)."""
import ctypes

import pytest

P = ctypes.c_void_p


def _lib():
    import paper_2503_21817_b200 as sk
    return sk.load_library()


def _cfg(hq=32, hk=8, d=128, dtype=0, causal=1, path=0, scale=0.1):
    from paper_2503_21817_b200.binding import _AttentionConfig
    return _AttentionConfig(hq, hk, d, dtype, causal, path, scale)


def _offsets(*v):
    return (ctypes.c_int32 * len(v))(*v)


@pytest.mark.parametrize("bad", [dict(hq=0), dict(hk=0), dict(hq=10, hk=4), dict(d=0), dict(d=12), dict(d=136), dict(dtype=2),
                                 dict(causal=2), dict(path=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(hq=65, hk=1)])
def test_attention_config_refused(bad):
    lib, cu, h = _lib(), _offsets(0, 10), P()
    cfg = _cfg(**bad)
    assert lib.skipffn_attention_plan_bytes(ctypes.byref(cfg), cu, 1) == 0
    want = 2 if bad in (dict(d=12), dict(d=136), dict(hq=65, hk=1)) else 1
    assert lib.skipffn_attention_create(ctypes.byref(h), ctypes.byref(cfg), cu, 1, P(4096), 1 << 30, None) == want
    assert not h.value


@pytest.mark.parametrize("cu", [(1, 5), (0, 5, 4), (0, 2 ** 31 - 1)])
def test_attention_offsets_refused(cu):
    lib, h, cfg = _lib(), P(), _cfg()
    arr = _offsets(*cu)
    assert lib.skipffn_attention_plan_bytes(ctypes.byref(cfg), arr, len(cu) - 1) == 0
    assert lib.skipffn_attention_create(ctypes.byref(h), ctypes.byref(cfg), arr, len(cu) - 1, P(4096), 1 << 40, None) in (1, 2)


def test_attention_plan_sizes_and_memory_checks():
    lib, h, cfg = _lib(), P(), _cfg()
    size = lambda c, *cu: lib.skipffn_attention_plan_bytes(ctypes.byref(c), _offsets(*cu), len(cu) - 1)
    # 32 tokens per 128-row tile (4 heads a group): 100 tokens = 2 forward pairs, 4 row tiles, 1 key tile
    assert size(cfg, 0, 100) == 256 + (2 + 4 + 1) * 16
    assert size(cfg, 0) == size(cfg, 0, 0, 0) == 256
    # a sequence never shares a tile with the next one
    assert size(cfg, 0, 50, 100) == 256 + (2 + 4 + 2) * 16
    # 64-row tiles of the plain-FMA kernels: 16 tokens each
    assert size(_cfg(dtype=1), 0, 100) == 256 + (7 + 7 + 2) * 16
    cu = _offsets(0, 100)
    create = lib.skipffn_attention_create
    assert create(ctypes.byref(h), ctypes.byref(cfg), cu, 1, None, 1 << 20, None) == 1
    assert create(ctypes.byref(h), ctypes.byref(cfg), cu, 1, P(4096 + 8), 1 << 20, None) == 1
    assert create(ctypes.byref(h), ctypes.byref(cfg), cu, 1, P(4096), 100, None) == 3
    assert create(ctypes.byref(h), ctypes.byref(cfg), cu, -1, P(4096), 1 << 20, None) == 1
    assert create(ctypes.byref(h), ctypes.byref(cfg), None, 1, P(4096), 1 << 20, None) == 1
    assert create(None, ctypes.byref(cfg), cu, 1, P(4096), 1 << 20, None) == 1
    assert lib.skipffn_attention_scratch_bytes(None) == 0 and lib.skipffn_attention_poll(None, None, None) == 1
    assert lib.skipffn_attention_forward(None, *[P(4096), 4096] * 4, P(4096), None) == 1


def test_layernorm_arguments_refused():
    lib = _lib()
    a, b, c = P(1 << 20), P(2 << 20), P(3 << 20)
    f = lambda x=a, g=b, be=None, n=4, C=64, dt=0, eps=1e-5, y=c: lib.skipffn_layernorm_forward(x, g, be, n, C, dt, eps, y, None, None, None)
    assert f(x=None) == f(g=None) == f(y=None) == f(n=-1) == f(C=0) == f(dt=2) == f(eps=-1.0) == f(eps=float("nan")) == 1
    assert f(x=P((1 << 20) + 8)) == f(y=P((3 << 20) + 8)) == f(be=P(4)) == 1
    assert f(C=12) == f(C=16392) == 2
    assert f(y=P((1 << 20) + 16)) == 1                          # partial overlap
    g = lambda dy=a, x=b, n=4, C=64, dx=c, sc=P(4 << 20), nb=1 << 24, m=P(5 << 20): lib.skipffn_layernorm_backward(
        dy, x, P(6 << 20), m, m, n, C, 0, dx, None, None, 0, sc, nb, None)
    assert g(dy=None) == g(dx=None) == g(sc=None) == g(m=None) == g(dx=P((1 << 20) + 32)) == g(dx=P((2 << 20) - 16)) == 1
    assert g(nb=100) == 3 and g(C=20) == 2
    assert lib.skipffn_layernorm_scratch_bytes(0) == 0 and lib.skipffn_layernorm_scratch_bytes(64) == 160 * 2 * 64 * 4


def test_layernorm_overlaps_and_alignment_refused():
    # every output on top of every other array of the call, but for the two pairs that may coincide
    lib = _lib()
    fwd = dict(x=1 << 20, gamma=2 << 20, beta=3 << 20, y=4 << 20, mean=5 << 20, rstd=6 << 20)
    f = lambda **kw: (lambda a: lib.skipffn_layernorm_forward(P(a["x"]), P(a["gamma"]), P(a["beta"]), 4, 64, 0, 1e-5, P(a["y"]),
                                                               P(a["mean"]), P(a["rstd"]), None))({**fwd, **kw})
    for o in ("y", "mean", "rstd"):
        for i in fwd:
            if i != o and (o, i) != ("y", "x"):
                assert f(**{o: fwd[i]}) == 1, (o, i)
    assert f(mean=fwd["mean"] + 2) == f(rstd=fwd["rstd"] + 1) == 1
    bwd = dict(dy=1 << 20, x=2 << 20, gamma=3 << 20, mean=4 << 20, rstd=5 << 20, dx=6 << 20, dgamma=7 << 20, dbeta=8 << 20, scratch=9 << 20)
    b = lambda dw=0, **kw: (lambda a: lib.skipffn_layernorm_backward(
        P(a["dy"]), P(a["x"]), P(a["gamma"]), P(a["mean"]), P(a["rstd"]), 4, 64, 0, P(a["dx"]), P(a["dgamma"]), P(a["dbeta"]), dw,
        P(a["scratch"]), 1 << 24, None))({**bwd, **kw})
    for o in ("dx", "dgamma", "dbeta", "scratch"):
        for i in bwd:
            if i != o and (o, i) not in (("dx", "dy"), ("dx", "x")):
                assert b(**{o: bwd[i]}) == 1, (o, i)
    assert b(dgamma=bwd["dgamma"] + 1) == b(dw=1, dbeta=bwd["dbeta"] + 2) == 1


def test_no_cpu_path():
    import torch
    import paper_2503_21817_b200 as sk
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(RuntimeError):
        sk.PackedAttention([0, 4], 1, 1, 64)
    with pytest.raises(ValueError):
        sk.layernorm_forward(torch.zeros(2, 8), torch.ones(8))
