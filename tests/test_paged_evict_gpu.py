"""Eviction from a paged cache on the GPU: rows, order and bytes exactly as the statement says."""
import numpy as np
import pytest

from cache_util import Batch, normal, within
from gpu_util import to_host
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def _weights(seed, n_seq, hk, width, kind="spread"):
    import torch
    g = torch.Generator().manual_seed(seed)
    if kind == "ties":
        w = torch.randint(0, 4, (n_seq, hk, width), generator=g).float()
    elif kind == "odd":                                          # signs, zeros of both signs, infinities, NaN
        w = torch.randn(n_seq, hk, width, generator=g)
        for x in (0.0, -0.0, float("inf"), -float("inf"), float("nan"), 1e-40, -1e-40):
            w[torch.rand(n_seq, hk, width, generator=g) < 0.1] = x
    else:
        w = torch.exp(2 * torch.randn(n_seq, hk, width, generator=g))
    return w.cuda()


def _expect(x, w, budget, sinks, recent):
    """(kept, new lens) by the statement."""
    w = w.cpu().numpy()
    kept = np.full((len(x.lens), x.hk, budget), -1, dtype=np.int32)
    for s, n in enumerate(x.lens):
        for h in range(x.hk):
            rows = oc.evict(w[s, h], n, budget, sinks, recent)
            kept[s, h, :len(rows)] = rows
    return kept, [min(n, budget) for n in x.lens]


def _same_bits(a, b):
    import torch
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype,order", [("bf16", "page,row,head"), ("fp32", "page,head,row"), ("bf16", "rows of both")])
@pytest.mark.parametrize("lens,budget,sinks,recent,kind,hk,d,page", [
    ((1,), 1, 0, 0, "spread", 1, 8, 8),                    # one row
    ((5, 0, 3), 4, 1, 2, "spread", 2, 64, 8),               # one to evict, no rows, all kept
    ((100, 300), 300, 0, 0, "spread", 2, 64, 16),           # nothing to evict
    ((700, 65, 64, 63), 64, 4, 16, "spread", 2, 64, 16),
    ((700, 200), 50, 0, 0, "ties", 3, 40, 24),              # many equal weights
    ((900, 333), 100, 10, 90, "spread", 2, 64, 16),         # protected rows alone
    ((900, 333), 100, 0, 100, "spread", 2, 64, 16),
    ((500, 90), 77, 3, 5, "odd", 2, 128, 8),
    ((9000,), 1500, 4, 128, "spread", 2, 128, 64),          # several steps of the move
    (tuple(20 + 13 * i % 90 for i in range(80)), 40, 2, 8, "ties", 4, 64, 16),   # many pairs: small clusters
])
def test_rows_kept_and_moved(lens, budget, sinks, recent, kind, hk, d, page, dtype, order):
    import torch
    import paper_2503_21817_b200 as sk
    x = Batch(sum(lens), [0] * len(lens), lens, hk, hk, d, page, dtype, order)
    w = _weights(len(lens) + budget, len(lens), hk, max(lens) + 3, kind)
    kept, new = _expect(x, w, budget, sinks, recent)
    y = Batch(1, [0] * len(lens), new, hk, hk, d, page, dtype)   # other pages; what is written is compared as a whole
    rows = {}
    for s in range(len(lens)):
        for name, t in (("k", x.k), ("v", x.v)):
            j = torch.arange(lens[s], device="cuda")
            rows[name, s] = t[torch.from_numpy(x.table[s]).cuda().long()[j // page], j % page].clone()
    moved = [t.clone() for t in (y.k, y.v)]
    in_place = [t.clone() for t in (x.k, x.v)]
    for s in range(len(lens)):
        for h in range(hk):
            for r, j in enumerate(kept[s, h][kept[s, h] >= 0]):
                for t, u, name in ((moved[0], in_place[0], "k"), (moved[1], in_place[1], "v")):
                    t[int(y.table[s, r // page]), r % page, h] = rows[name, s][int(j), h]
                    u[int(x.table[s, r // page]), r % page, h] = rows[name, s][int(j), h]
    want_w = np.zeros((len(lens), hk, budget), dtype=np.float32)
    for s in range(len(lens)):
        for h in range(hk):
            m = new[s]
            want_w[s, h, :m] = w.cpu().numpy()[s, h, kept[s, h, :m]]
    copies = x.k.clone(), x.v.clone()
    for into in (y.cache, None, x.cache):                        # its own object: in place, too
        if into is x.cache:
            x.k.copy_(copies[0]), x.v.copy_(copies[1])
        got, got_lens, got_w = x.cache.evict(w, budget, sinks=sinks, recent=recent, into=into)
        x.cache.poll()
        assert np.array_equal(got.cpu().numpy(), kept)
        assert got_lens.tolist() == new
        assert np.array_equal(got_w.cpu().numpy(), want_w, equal_nan=True)
        a, b = (y.k, y.v) if into is y.cache else (x.k, x.v)
        c, e = moved if into is y.cache else in_place
        assert _same_bits(a, c) and _same_bits(b, e)


def test_other_stream_and_replay():
    import torch
    x = Batch(3, [0, 0], (800, 90), 2, 2, 64, 16)
    y = Batch(4, [0, 0], (100, 90), 2, 2, 64, 16)
    w = _weights(5, 2, 2, 800)
    want = x.cache.evict(w, 100, 2, 20, into=y.cache)
    pages = y.k.clone(), y.v.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = x.cache.evict(w, 100, 2, 20, into=y.cache)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = x.cache.evict(w, 100, 2, 20, into=y.cache)
    other = _weights(6, 2, 2, 800)
    keep = w.clone()
    for v in (other, keep):
        w.copy_(v)
        y.k.fill_(0.0), y.v.fill_(0.0)
        graph.replay()
        kept, _ = _expect(x, v, 100, 2, 20)
        assert np.array_equal(res[0].cpu().numpy(), kept)
    assert all(torch.equal(a, b) for a, b in zip(want, res))
    m = [torch.arange(n, device="cuda") for n in (100, 90)]
    for s in range(2):
        p = y.d_table[s].long()[m[s] // 16]
        assert _same_bits(y.k[p, m[s] % 16], pages[0][p, m[s] % 16]) and _same_bits(y.v[p, m[s] % 16], pages[1][p, m[s] % 16])


def test_wrong_integers_are_reported():
    import torch
    import paper_2503_21817_b200 as sk
    x = Batch(7, [0, 0], (200, 90), 2, 2, 64, 16)
    y = Batch(8, [0, 0], (60, 60), 2, 2, 64, 16)
    w = _weights(9, 2, 2, 200)
    want = x.cache.evict(w, 60, into=y.cache)
    good = y.k[y.d_table[1, 0].long()].clone()

    def again(cache, site):
        res = x.cache.evict(w, 60, into=y.cache)
        with pytest.raises(sk.SkipFFNError, match=f"site {site}"):
            cache.poll()
        x.cache.poll(), y.cache.poll()
        return res

    x.d_table[0, 0] = -1
    kept, *_ = again(x.cache, 66)
    assert torch.equal(kept, want[0])
    page, row = y.d_table[1, 0].long(), torch.arange(16)
    assert _same_bits(y.k[page], good)
    x.d_table[0, 0] = int(x.table[0, 0])
    y.d_table[0, 1] = 10 ** 6
    again(y.cache, 66)
    y.d_table[0, 1] = int(y.table[0, 1])
    x.d_lens[0] = 10 ** 6
    again(x.cache, 65)
    x.d_lens[0] = 201                                            # rows that no weight belongs to
    again(x.cache, 68)
    x.d_lens[0] = 200
    # a destination with too little room
    z = Batch(8, [0, 0], (30, 30), 2, 2, 64, 16)
    kept, lens, _ = x.cache.evict(w, 60, into=z.cache)
    with pytest.raises(sk.SkipFFNError, match="site 67"):
        z.cache.poll()
    assert torch.equal(kept, want[0])


def test_from_prompt_to_answers():
    """What a decoder does: prompts through rotary positions into pages, attention, weights, eviction, new tokens."""
    import torch
    import paper_2503_21817_b200 as sk
    lens, hq, hk, d, page, budget = (180, 70), 8, 2, 64, 16, 64
    n_seq, steps = len(lens), 3
    x = Batch(11, lens, [m + steps for m in lens], hq, hk, d, page)
    x.k.fill_(float("nan")), x.v.fill_(float("nan"))
    rot = sk.RotaryQK(hq, hk, d, sections=[8, 12, 12])
    n = sum(lens)
    g = [1 + 0.2 * normal(i, d) for i in (1, 2)]
    inputs = [(normal(20 + i, m, hq, d), normal(30 + i, m, hk, d), normal(40 + i, m, hk, d)) for i, m in enumerate([n] + [n_seq] * steps)]
    pos = torch.randint(0, 500, (3, n), dtype=torch.int32, generator=torch.Generator().manual_seed(3)).cuda()
    x.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    # the prompt, and the same through the packed attention
    q = rot.append(x.cache, *inputs[0], pos, *g)
    out, lse = x.cache.attention(q)
    q2, k2 = rot.forward(inputs[0][0], inputs[0][1], pos, *g)
    packed = sk.PackedAttention([0, lens[0], n], hq, hk, d)
    o2, l2 = packed.forward(q2, k2, inputs[0][2])
    assert torch.equal(q, q2) and bool(((lse - l2).abs() < 1e-4).all())
    assert bool(((out.float() - o2.float()).abs() <= 2.0 ** -6 * (1 + o2.float().abs())).all())
    keys = [to_host(k2[a:b]) for a, b in ((0, lens[0]), (lens[0], n))]
    values = [to_host(inputs[0][2][a:b]) for a, b in ((0, lens[0]), (lens[0], n))]
    w = x.cache.weights(q, lse)
    r_w, e_w = oc.weights(to_host(q), keys, to_host(lse), [0, lens[0], n], lens, hk, d ** -0.5, w.shape[2])
    within(w, r_w, e_w, "weights")
    kept, new, w = x.cache.evict(w, budget, sinks=2, recent=8)
    rows = kept.cpu().numpy()
    held = []
    for s in range(n_seq):
        m = min(lens[s], budget)
        held.append([np.stack([t[s][rows[s, h, :m], h] for h in range(hk)], 1) for t in (keys, values)])
    # new tokens, one for each sequence at a time
    x.d_cu.copy_(torch.arange(n_seq + 1, dtype=torch.int32))
    for step in range(steps):
        x.d_lens.copy_(new + step + 1)
        p = torch.full((3, n_seq), 500 + step, dtype=torch.int32, device="cuda")
        q = rot.append(x.cache, *inputs[1 + step], p, *g)
        out, lse = x.cache.attention(q)
        _, k2 = rot.forward(inputs[1 + step][0], inputs[1 + step][1], p, *g)
        for s in range(n_seq):
            held[s] = [np.concatenate((held[s][0], to_host(k2[s:s + 1]))), np.concatenate((held[s][1], to_host(inputs[1 + step][2][s:s + 1])))]
        r_out, r_lse, e_out, e_lse = oc.attention(to_host(q), [t[0] for t in held], [t[1] for t in held], [0, 1, 2], [t[0].shape[0] for t in held],
                                                  d ** -0.5)
        within(out, r_out, e_out, "out")
        within(lse, r_lse, e_lse, "lse")
        x.cache.poll()
