"""Rotary positions with per-head norms on the GPU against their fp64 statement, every element within its bound."""
import numpy as np
import pytest

from cache_util import DT, Batch, normal, within
from gpu_util import to_host
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def _case(seed, n, hq, hk, d, dtype, axes=1, norm=True, fused=False, far=40000):
    import torch
    q, k, gq, gk = normal(seed, n, hq, d, dtype=dtype, std=2.0), normal(seed + 1, n, hk, d, dtype=dtype), normal(seed + 2, hq, d, dtype=dtype), None
    pos = torch.randint(-far, far, (axes, n), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()
    if fused:
        q, k, _ = torch.cat((q, k, k), 1).split((hq, hk, hk), 1)
    g = [normal(seed + i, d, dtype=dtype) for i in (5, 6)] if norm else [None, None]
    dq, dk = normal(seed + 7, n, hq, d, dtype=dtype), normal(seed + 8, n, hk, d, dtype=dtype)
    return q, k, pos, g, dq, dk


def _check(rot, q, k, pos, g, dq, dk, freq, axis, rotary_dim, inter, dtype, eps=1e-6, dw_fp32=False):
    P = pos.cpu().numpy()
    out = rot.forward(q, k, pos, *g)
    back = rot.backward(dq, dk, q, k, pos, *g, dw_fp32=dw_fp32)
    for i, (x, dy, name) in enumerate(((q, dq, "q"), (k, dk, "k"))):
        G = None if g[i] is None else to_host(g[i])
        y, e = oc.rotary_forward(to_host(x), P, freq, axis, rotary_dim, inter, G, eps, dtype)
        within(out[i], y, e, name)
        (dx, dg), (ex, eg) = oc.rotary_backward(to_host(dy), to_host(x), P, freq, axis, rotary_dim, inter, G, eps, dtype,
                                                "fp32" if dw_fp32 else None)
        within(back[i], dx, ex, "d" + name)
        if G is None:
            assert back[2 + i] is None
        else:
            within(back[2 + i], dg, eg, "dgamma_" + name)
    return out, back


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hq,hk,d,rot,axes,norm,inter", [
    (1, 1, 1, 8, 8, 1, True, False),               # the smallest row: one lane
    (1, 32, 8, 128, 128, 1, True, False),          # one token
    (37, 8, 2, 128, 128, 3, True, False),          # text / height / width
    (150, 4, 4, 64, 64, 2, False, False),          # vision tower
    (151, 5, 1, 96, 96, 1, True, True),            # 6 of 8 lanes of a row
    (9, 3, 3, 40, 40, 1, True, False),             # halves of 20 columns
    (65, 7, 1, 80, 32, 1, True, False),            # columns behind the rotated ones
    (33, 6, 2, 80, 24, 2, False, True),
    (20, 4, 2, 256, 256, 4, True, False),          # the widest head
    (20, 4, 2, 248, 128, 1, True, True),
    (50, 2, 1, 128, 0, 1, True, False),            # norm alone
    (1500, 12, 4, 64, 64, 1, True, False),         # many CTAs, several blocks each
])
def test_against_64_bits(n, hq, hk, d, rot, axes, norm, inter, dtype):
    import paper_2503_21817_b200 as sk
    q, k, pos, g, dq, dk = _case(n + d, n, hq, hk, d, dtype, axes, norm, fused=n % 2 == 1)
    r = np.random.default_rng(d)
    freq, axis = 10000.0 ** -r.random(rot // 2), np.sort(r.integers(0, axes, rot // 2))
    sections = [int((axis == a).sum()) for a in range(axes)]
    obj = sk.RotaryQK(hq, hk, d, rotary_dim=rot, sections=sections, inv_freq=freq, interleaved=inter)
    _check(obj, q, k, pos, g, dq, dk, freq, axis, rot, inter, dtype, dw_fp32=n % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_default_and_restarted_frequencies_and_far_positions(dtype):
    import torch
    import paper_2503_21817_b200 as sk
    q, k, pos, g, dq, dk = _case(3, 12, 4, 2, 64, dtype, 2)
    far = [0, 1, -1, 7, 2 ** 20 + 1, 2 ** 24 + 3, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 131071, -131072, 99999]
    pos = torch.tensor([far, far[::-1]], dtype=torch.int32, device="cuda")
    one = sk.RotaryQK(4, 2, 64, base=500000.0, sections=[8, 24])
    _check(one, q, k, pos, g, dq, dk, [500000.0 ** (-p / 32) for p in range(32)], [0] * 8 + [1] * 24, 64, False, dtype)
    two = sk.RotaryQK(4, 2, 64, base=100.0, sections=[16, 16], restart=True)
    _check(two, q, k, pos, g, dq, dk, [100.0 ** (-p / 16) for p in range(16)] * 2, [0] * 16 + [1] * 16, 64, False, dtype)


def test_no_tokens():
    import torch
    import paper_2503_21817_b200 as sk
    q, k, pos, g, dq, dk = _case(4, 5, 4, 2, 64, "bf16")
    rot = sk.RotaryQK(4, 2, 64)
    a = [t[:0] for t in (q, k)]
    out = rot.forward(*a, pos[:, :0], *g)
    back = rot.backward(dq[:0], dk[:0], *a, pos[:, :0], *g)
    assert out[0].shape == (0, 4, 64) and back[1].shape == (0, 2, 64) and not back[2].any() and not back[3].any()


def test_norm_of_small_and_zero_rows():
    import torch
    import paper_2503_21817_b200 as sk
    q, k, pos, g, dq, dk = _case(4, 6, 4, 2, 64, "fp32")
    q[1], q[2], k[3] = 0.0, q[2] * 1e-4, k[3] * 1e-18
    _check(sk.RotaryQK(4, 2, 64, eps=1e-5), q, k, pos, g, dq, dk, [10000.0 ** (-p / 32) for p in range(32)], [0] * 32, 64, False, "fp32", eps=1e-5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place_strided_results_other_stream_and_replay(dtype):
    import torch
    import paper_2503_21817_b200 as sk
    n, hq, hk, d = 301, 8, 2, 128
    q, k, pos, g, dq, dk = _case(5, n, hq, hk, d, dtype)
    rot = sk.RotaryQK(hq, hk, d)
    want, grads = rot.forward(q, k, pos, *g), rot.backward(dq, dk, q, k, pos, *g)
    both = torch.full((n, hq + 2 * hk, d), 3.0, dtype=DT[dtype], device="cuda")
    a, b, rest = both.split((hq, hk, hk), 1)
    a.copy_(q), b.copy_(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rot.forward(a, b, pos[0], *g, out_q=a, out_k=b)             # in place, slices of one projection
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and bool((rest == 3.0).all())
    # gradients over the upstream ones, and over the inputs
    a.copy_(dq), b.copy_(dk)
    got = rot.backward(a, b, q, k, pos, *g, dq=a, dk=b)
    assert all(torch.equal(x, y) for x, y in zip(grads, got))
    a.copy_(q), b.copy_(k)
    got = rot.backward(dq, dk, a, b, pos, *g, dq=a, dk=b)
    assert all(torch.equal(x, y) for x, y in zip(grads, got))
    held = [t.clone() for t in (q, k, dq, dk)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = (*rot.forward(held[0], held[1], pos, *g), *rot.backward(held[2], held[3], held[0], held[1], pos, *g))
    for _ in range(2):
        for t in res:
            t.zero_()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(res, (*want, *grads)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("order", ["page,row,head", "page,head,row", "pages of both", "rows of both"])
def test_append_writes_the_rows_of_the_new_tokens_and_nothing_else(order, dtype):
    import torch
    import paper_2503_21817_b200 as sk
    new, lens, hq, hk, d, page = (1, 0, 5, 17, 2), (1, 9, 24, 20, 2), 8, 2, 64, 8
    pad, n = 3, 25
    q, k, pos, g, *_ = _case(6, n + pad, hq, hk, d, dtype)
    v = normal(9, n + pad, hk, d, dtype=dtype)
    x = Batch(6, new, lens, hq, hk, d, page, dtype, order)
    before = x.k.clone(), x.v.clone()
    rot = sk.RotaryQK(hq, hk, d)
    want = rot.forward(q, k, pos, *g)
    out = torch.full_like(want[0], 7.0)
    rot.append(x.cache, q, k, v, pos, *g, out_q=out)
    x.cache.poll()
    assert torch.equal(out[:n], want[0][:n]) and bool((out[n:] == 7.0).all())
    for plain in (False, True):
        if plain:                                                # the form without rotation
            x.k.copy_(before[0]), x.v.copy_(before[1])
            x.cache.append(k, v)
        expect = before[0].clone(), before[1].clone()
        for s, (m, length) in enumerate(zip(new, lens)):
            for i in range(m):
                j = length - m + i
                at = int(x.table[s, j // page]), j % page
                expect[0][at], expect[1][at] = (k if plain else want[1])[x.cu[s] + i], v[x.cu[s] + i]
        assert torch.equal(x.k.nan_to_num(9.0), expect[0].nan_to_num(9.0)) and torch.equal(x.v.nan_to_num(9.0), expect[1].nan_to_num(9.0))


def test_append_to_many_sequences_finds_each():
    # 1500 sequences, some without new tokens: the search over the offsets takes three steps
    import torch
    new = [i % 3 for i in range(1500)]
    lens = [max(m, 1) for m in new]
    x = Batch(8, new, lens, 1, 1, 8, 8, "fp32")
    n = x.cu[-1]
    k, v = normal(1, n, 1, 8, dtype="fp32"), normal(2, n, 1, 8, dtype="fp32")
    x.cache.append(k, v)
    x.cache.poll()
    for s in range(0, 1500, 7):
        page = int(x.table[s, 0])
        assert torch.equal(x.k[page, :new[s]], k[x.cu[s]:x.cu[s + 1]]) and torch.equal(x.v[page, :new[s]], v[x.cu[s]:x.cu[s + 1]])


def test_append_without_room_or_to_a_page_that_is_not_there():
    import torch
    import paper_2503_21817_b200 as sk
    x = Batch(11, (3, 2, 4), (3, 2, 4), 2, 2, 8, 8, "fp32")
    k, v = normal(1, 9, 2, 8, dtype="fp32"), normal(2, 9, 2, 8, dtype="fp32")
    for lens, first, site in (((3, 1, 4), int(x.table[1, 0]), 67), ((3, 2, 4), 1 << 20, 66), ((3, 2, 4), -5, 66)):
        x.k.fill_(7.0)
        x.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        x.d_table[1, 0] = first
        x.cache.append(k, v)
        with pytest.raises(sk.SkipFFNError, match=f"site {site}"):
            x.cache.poll()
        x.cache.poll()                                           # reported once
        assert torch.equal(x.k[int(x.table[0, 0]), :3], k[:3]) and torch.equal(x.k[int(x.table[2, 0]), :4], k[5:])
        if site == 67:
            assert torch.equal(x.k[int(x.table[1, 0]), 0], k[4]) and bool((x.k[int(x.table[1, 0]), 1:] == 7.0).all())
        else:
            assert bool((x.k[int(x.table[1, 0])] == 7.0).all())
