"""Attention over a paged cache and the weights of its rows on the GPU against their fp64 statements."""
import numpy as np
import pytest

from cache_util import Batch, normal, within
from gpu_util import to_host
from oracle import cache as oc

pytestmark = pytest.mark.gpu

CASES = [
    # new, lens, hq, hk, d, page
    ((1,), (1,), 4, 1, 128, 16),                            # one token, one row
    ((1, 1, 1, 1), (15, 16, 17, 64), 8, 2, 128, 16),        # around a page and a block
    ((1, 1, 1), (63, 65, 300), 2, 2, 64, 8),
    ((1, 0, 1, 0), (5, 7, 0, 0), 4, 2, 64, 24),             # nothing new; no rows at all; pages of 24 rows
    ((3, 1, 4), (2, 1, 40), 4, 2, 64, 8),                   # more new tokens than rows: the first see nothing
    ((2, 5, 3), (130, 70, 9), 8, 2, 128, 32),               # 20 rows: two groups of warps
    ((9, 16, 1), (200, 16, 77), 8, 2, 96, 16),              # 64 rows, 96 columns
    ((1, 1), (90, 400), 40, 1, 128, 64),                    # one kv head for 40
    ((1, 1), (90, 129), 64, 1, 40, 16),                     # a group of 64, 40 columns
    ((1,), (5000,), 8, 2, 80, 16),                          # one sequence over all SMs, 80 columns
    ((1,) * 150, tuple(1 + 37 * i % 200 for i in range(150)), 4, 2, 64, 16),   # more sequences than threads of a CTA
    ((17,), (17,), 8, 2, 128, 16),                          # a chunk that is the whole prompt
    ((100, 1, 33, 0, 1), (300, 50, 33, 10, 700), 8, 2, 128, 16),   # chunks and single tokens
    ((300,), (1100,), 12, 4, 64, 48),                       # pages that end inside a tile
    ((130, 70), (130, 200), 4, 4, 128, 128),
    ((128, 129, 127), (128, 129, 400), 2, 2, 64, 64),       # around a tile of one head
    ((70, 40), (71, 45), 10, 2, 80, 16),                    # groups of 5
    ((50, 60), (20, 60), 4, 2, 128, 8),                     # a chunk whose first tokens see nothing
    ((20,), (100,), 64, 1, 32, 16),
    ((150,) * 8, (150, 160, 170, 180, 190, 200, 210, 220), 32, 1, 64, 16),     # several tiles for every CTA
    ((5, 7, 16), (1500, 40, 900), 8, 2, 64, 16),            # 20 to 64 rows over many blocks
]


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("new,lens,hq,hk,d,page", CASES)
def test_attention_and_weights_against_64_bits(new, lens, hq, hk, d, page, dtype, path):
    import torch
    x = Batch(sum(lens), new, lens, hq, hk, d, page, dtype, path=path)
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    r_out, r_lse, e_out, e_lse = x.want()
    within(out, r_out, e_out, "out")
    within(lse, r_lse, e_lse, "lse")
    width = max(lens) + 5
    prior = torch.rand(len(lens), hk, width, device="cuda")
    w = x.cache.weights(x.q, lse, prior=prior)
    x.cache.poll()
    r_w, e_w = oc.weights(to_host(x.q), x.keys, to_host(lse), x.cu, lens, hk, x.scale, width, to_host(prior))
    within(w, r_w, e_w, "weights")
    # the same bits again, weights over their prior
    out2, lse2 = x.cache.attention(x.q)
    w2 = x.cache.weights(x.q, lse, prior=prior, out=prior)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(w, w2) and w2 is prior


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("order", ["page,head,row", "pages of both", "rows of both"])
def test_memory_orders_of_the_pages(order, dtype):
    for new, lens in (((1, 1, 2), (70, 9, 130)), ((40, 1, 2), (70, 9, 130))):
        x = Batch(1, new, lens, 8, 2, 64, 16, dtype, order)
        out, lse = x.cache.attention(x.q)
        r_out, r_lse, e_out, e_lse = x.want()
        within(out, r_out, e_out, "out")
        r_w, e_w = oc.weights(to_host(x.q), x.keys, to_host(lse), x.cu, lens, 2, x.scale, 130)
        within(x.cache.weights(x.q, lse, width=130), r_w, e_w, "weights")
        x.cache.poll()


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
def test_large_scores_and_other_scales(dtype, path):
    # scores up to some hundreds: the running maximum moves block by block, the sums must follow
    for new, lens in (((1, 3), (400, 129)), ((40, 100), (400, 129))):
        x = Batch(2, new, lens, 8, 2, 64, 16, dtype, path=path)
        for scale in (2.0, 0.01):
            out, lse = x.cache.attention(x.q, scale=scale)
            r_out, r_lse, e_out, e_lse = x.want(scale)
            within(out, r_out, e_out, "out")
            within(lse, r_lse, e_lse, "lse")


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("new", [(1, 2, 1), (60, 2, 1), (60, 33, 40)])
def test_neighbours_unowned_rows_and_rows_behind_the_batch(new, dtype, path):
    # what no row of a sequence owns is NaN from the start; here the neighbours' rows become it too
    import torch
    lens, pad = (90, 45, 130), 5
    x = Batch(3, new, lens, 8, 2, 64, 24, dtype, pad=pad, path=path)
    n = x.cu[-1]
    out, lse = x.cache.attention(x.q)
    w = x.cache.weights(x.q, lse.nan_to_num(0.0), width=130)
    for s in (0, 2):
        for p in x.table[s][x.table[s] >= 0]:
            x.k[int(p)] = float("inf")
            x.v[int(p)] = float("nan")
    x.q[:x.cu[1]] = float("nan")
    x.q[x.cu[2]:] = float("nan")
    out2, lse2 = x.cache.attention(x.q, out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0))
    w2 = x.cache.weights(x.q, lse.nan_to_num(0.0), width=130)
    x.cache.poll()
    a, b = x.cu[1], x.cu[2]
    assert torch.equal(out[a:b], out2[a:b]) and torch.equal(lse[a:b], lse2[a:b]) and torch.equal(w[1], w2[1])
    assert bool((out2[n:] == 7.0).all()) and bool((lse2[n:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths_offsets_and_pages_that_follow_a_replayed_graph(dtype):
    import torch
    hq, hk, d, page = 8, 2, 64, 16
    for new, lens, new2, lens2 in (((1, 1, 1), (40, 100, 7), (1, 1, 1), (41, 101, 8)), ((50, 1, 0), (90, 100, 7), (2, 48, 1), (41, 101, 8))):
        a, b = (Batch(s, m, l, hq, hk, d, page, dtype, max_new=50) for s, m, l in ((4, new, lens), (5, new2, lens2)))
        x = Batch(4, new, lens, hq, hk, d, page, dtype, max_new=50)
        x.cache.attention(x.q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = x.cache.attention(x.q)
        for y in (a, b, a):
            pages = min(x.k.shape[0], y.k.shape[0])
            assert max(y.table.max(), 0) < pages and y.table.shape == x.table.shape and y.q.shape == x.q.shape
            x.k[:pages].copy_(y.k[:pages]), x.v[:pages].copy_(y.v[:pages]), x.q.copy_(y.q)
            x.d_table.copy_(y.d_table), x.d_cu.copy_(y.d_cu), x.d_lens.copy_(y.d_lens)
            graph.replay()
            r_out, r_lse, e_out, e_lse = y.want()
            within(out, r_out, e_out, "out")
            within(lse, r_lse, e_lse, "lse")
        x.cache.poll()


@pytest.mark.parametrize("new", [(1, 1, 2), (70, 1, 40)])
def test_calls_on_two_streams_at_once_and_two_graphs(new):
    import torch
    x = Batch(6, new, (3000, 900, 2000), 8, 2, 128, 16)
    q2 = normal(77, *x.q.shape)
    want = [x.cache.attention(q) for q in (x.q, q2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    res = []
    for _ in range(4):
        for s, q in zip(streams, (x.q, q2)):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                res.append(x.cache.attention(q))
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(res):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])
    graphs = []
    for q in (x.q, q2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = x.cache.attention(q)
        graphs.append((g, r))
    for _ in range(3):
        for s, (g, r) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for (g, r), w in zip(graphs, want):
        assert torch.equal(r[0], w[0]) and torch.equal(r[1], w[1])
    x.cache.poll()


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("new", [(1, 2, 1), (60, 33, 40)])
def test_wrong_integers_are_reported_and_leave_the_other_sequences_alone(new, dtype, path):
    import torch
    import paper_2503_21817_b200 as sk
    lens = (90, 45, 130)
    x = Batch(7, new, lens, 4, 2, 64, 16, dtype, path=path)      # the table's unused entries are -1
    out, lse = x.cache.attention(x.q)
    w = x.cache.weights(x.q, lse, width=130)
    good = x.d_table.clone(), x.d_cu.clone(), x.d_lens.clone()
    a, b = x.cu[1], x.cu[2]

    def again(site, which=(0, 2), weigh=True):
        o, l = x.cache.attention(x.q, out=torch.zeros_like(out), lse=torch.zeros_like(lse))
        with pytest.raises(sk.SkipFFNError, match=f"site {site}"):
            x.cache.poll()
        if weigh:
            w2 = x.cache.weights(x.q, lse, width=130)
            with pytest.raises(sk.SkipFFNError, match=f"site {site}"):
                x.cache.poll()
        x.cache.poll()
        for s in which:
            r = slice(x.cu[s], x.cu[s + 1])
            assert torch.equal(o[r], out[r]) and torch.equal(l[r], lse[r])
            assert not weigh or torch.equal(w2[s], w[s])
        for t, g in zip((x.d_table, x.d_cu, x.d_lens), good):
            t.copy_(g)

    for page in (-1, -2 ** 31, x.k.shape[0], 2 ** 31 - 1):       # a page that does not exist
        x.d_table[1, 1] = page
        again(66)
    for length in (-3, 10 ** 6, 2 ** 31 - 1):                    # lengths that the table has no room for
        x.d_lens[1] = length
        again("65" if length < 0 else "6[56]")                   # cut to the table's width it reaches pages that are not there, too
    x.d_cu[3] = 2 ** 31 - 1                                      # offsets past the call's tokens
    again(64, (0, 1))
    x.d_cu[1] = -5                                               # descending
    again(64, (2,))
    x.d_cu.copy_(torch.tensor([0, 0, 0, x.cu[-1]], dtype=torch.int32))   # more new tokens than max_new
    if x.cu[-1] > max(new):
        again(64, ())
    else:
        x.d_cu.copy_(good[1])


def test_weights_of_more_rows_than_their_width_are_reported():
    import paper_2503_21817_b200 as sk
    x = Batch(8, (1,), (50,), 2, 2, 64, 16)
    _, lse = x.cache.attention(x.q)
    full = x.cache.weights(x.q, lse, width=64)
    x.cache.poll()
    part = x.cache.weights(x.q, lse, width=20)
    with pytest.raises(sk.SkipFFNError, match="site 68"):
        x.cache.poll()
    assert bool((part == full[..., :20]).all())


@pytest.mark.parametrize("new,lens,hq,hk,d,page", [
    ((130, 1, 70), (2500, 3000, 1200), 8, 8, 64, 16),        # several units for every CTA, of one and of several steps
    ((90,), (30000,), 4, 1, 128, 64),
    ((40, 200), (9000, 9001), 16, 4, 64, 32),
])
def test_weights_with_several_units_and_steps_per_cta(new, lens, hq, hk, d, page):
    # small heads so that the statement in 64 bits stays quick; the logarithms are any numbers near the right ones
    import torch
    x = Batch(12, new, lens, hq, hk, d, page)
    lse = torch.randn(x.cu[-1], hq, generator=torch.Generator().manual_seed(1)).cuda() + 8.0
    lse[3] = float("-inf")
    w = x.cache.weights(x.q, lse, width=max(lens))
    x.cache.poll()
    r_w, e_w = oc.weights(to_host(x.q), x.keys, to_host(lse), x.cu, lens, hk, x.scale, max(lens))
    within(w, r_w, e_w, "weights")


def test_long_cache_rows_against_64_bits():
    x = Batch(9, (1, 70), (70001, 9000), 4, 1, 128, 64)
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    r_out, r_lse, e_out, e_lse = x.want()
    within(out, r_out, e_out, "out")
    within(lse, r_lse, e_lse, "lse")


@pytest.mark.parametrize("new", [(1, 3), (50, 3)])
def test_pages_past_four_gigabytes(new):
    # 40 000 pages of 64 rows: 5.2 GB for the keys alone; the sequences' pages are the last ones
    import torch
    import paper_2503_21817_b200 as sk
    lens, hq, hk, d, page, pages = (200, 100), 8, 8, 128, 64, 40000
    x = Batch(13, new, lens, hq, hk, d, page, spare=0)
    k, v = (torch.empty(pages, page, hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    shift = pages - x.k.shape[0]
    k[shift:], v[shift:] = x.k, x.v
    table = torch.where(x.d_table >= 0, x.d_table + shift, x.d_table)
    far = sk.PagedCache(k, v, table, x.d_cu, x.d_lens, max(new))
    out, lse = far.attention(x.q)
    want, lse2 = x.cache.attention(x.q)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    w = far.weights(x.q, lse, width=200)
    assert torch.equal(w, x.cache.weights(x.q, lse, width=200))
    n = x.cu[-1]
    nk, nv = normal(1, n, hk, d), normal(2, n, hk, d)
    far.append(nk, nv), x.cache.append(nk, nv)
    kept = far.evict(w, 64, 2, 8)
    assert all(torch.equal(a, b) for a, b in zip(kept, x.cache.evict(w, 64, 2, 8)))
    far.poll(), x.cache.poll()
    for a, b in ((k[shift:], x.k), (v[shift:], x.v)):
        assert torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def test_no_tokens_no_sequences_no_pages():
    import torch
    import paper_2503_21817_b200 as sk
    x = Batch(14, (1, 1), (20, 30), 4, 2, 64, 16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q0 = x.q[:0]
    assert x.cache.attention(q0)[0].shape == (0, 4, 64)
    none = sk.PagedCache(x.k, x.v, x.d_table[:0], i32(0), i32(), 1)
    out, lse = none.attention(x.q, out=torch.full_like(x.q, 7.0))
    assert bool((out == 7.0).all()) and none.weights(x.q, lse, width=9).shape == (0, 2, 9)
    empty = sk.PagedCache(x.k[:0], x.v[:0], x.d_table[:, :0], x.d_cu, i32(0, 0), 1)
    for new in (1, 60):                                          # the kernel for few rows, the one for chunks
        e = sk.PagedCache(x.k[:0], x.v[:0], x.d_table[:, :0], i32(0, 0, new), i32(0, 0), new)
        q = normal(5, new, 4, 64)
        out, lse = e.attention(q)
        assert bool((out == 0).all()) and bool((lse == float("-inf")).all())
        e.poll()
    w = empty.weights(x.q, lse[:2], width=5)
    assert bool((w == 0).all())
    kept, lens, ww = empty.evict(w, 3)
    assert bool((kept == -1).all()) and lens.tolist() == [0, 0] and bool((ww == 0).all())
    empty.poll()


def test_a_key_that_scores_minus_infinity_has_probability_zero():
    import torch
    for new in ((1,), (40,)):
        x = Batch(10, new, (200,), 2, 1, 64, 16)
        x.q.abs_()
        page = x.d_table[0].long()
        for j in (*range(0, 64), 100, 150):
            x.k[page[j // 16], j % 16] = float("-inf")
        x.keys[0][[*range(0, 64), 100, 150]] = -1e30
        out, lse = x.cache.attention(x.q)
        n = new[0]
        k, v, q = x.keys[0][:, 0], x.values[0][:, 0], to_host(x.q)
        for i in range(n):
            for h in range(2):
                s = x.scale * (k[:200 - n + i + 1] @ q[i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                assert np.allclose(to_host(out)[i, h], p @ v[:p.size], atol=2.0 ** -7 * np.abs(v).max())


@pytest.mark.parametrize("tokens,lens,hq,hk,d", [
    (8, range(129, 729, 4), 8, 2, 128),                      # 32 rows, 2 to 6 blocks, most of them within one run
    (30, range(30, 780, 5), 4, 1, 64),                       # 120 rows, 1 to 7 blocks
    (17, (257, 384, 385, 1000), 2, 2, 80),                   # 17 rows, all of them cut
])
def test_sequences_of_one_row_tile_over_several_blocks(tokens, lens, hq, hk, d):
    import torch
    lens = list(lens)
    x = Batch(14, (tokens,) * len(lens), lens, hq, hk, d, 16)
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    r_out, r_lse, e_out, e_lse = x.want()
    within(out, r_out, e_out, "out")
    within(lse, r_lse, e_lse, "lse")
    # every other block scores minus infinity: half of a tile's blocks leave nothing, then the other half
    for odd in (0, 1):
        y = Batch(14, (tokens,) * len(lens), lens, hq, hk, d, 16)
        y.q.abs_()
        for s, n in enumerate(lens):
            j = torch.arange(n, device="cuda")
            j = j[j // 128 % 2 == odd]
            y.k[y.d_table[s].long()[j // 16], j % 16] = float("-inf")
            y.keys[s][j.cpu().numpy()] = -1e30
        out, lse = y.cache.attention(y.q)
        y.cache.poll()
        q = to_host(y.q)
        for s, n in enumerate(lens):
            for i in (0, tokens - 1):
                t, h = s * tokens + i, hq - 1
                seen = np.arange(n - tokens + i + 1)
                seen = seen[seen // 128 % 2 != odd]
                if not seen.size:
                    assert bool((out[t, h] == 0).all()) and lse[t, h].item() == float("-inf")
                    continue
                sc = y.scale * (y.keys[s][seen, h // (hq // hk)] @ q[t, h])
                p = np.exp(sc - sc.max())
                v = y.values[s][seen, h // (hq // hk)]
                # weights and the result in bf16: half a step each, of values of at most the largest
                assert np.allclose(to_host(out[t, h]), p / p.sum() @ v, rtol=0, atol=2.0 ** -7 * np.abs(v).max())
                assert abs(lse[t, h].item() - sc.max() - np.log(p.sum())) < 1e-4 * max(1.0, abs(sc.max()))


@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("new,lens,hq,hk,d", [
    ((1, 2, 0, 1), (9, 300, 8, 1), 1, 1, 128),               # 1 and 2 rows
    ((3, 1, 2), (3, 500, 77), 1, 1, 40),                     # up to 4
    ((1, 1), (2000, 17), 4, 1, 64),
    ((1, 2, 1), (129, 7, 640), 6, 2, 72),                    # up to 6
    ((8, 5), (8, 1000), 1, 1, 128),
    ((2, 30, 1, 3), (200, 31, 900, 150), 4, 1, 96),          # 8 and fewer beside 12 and 120
    ((3, 1), (2, 16), 2, 1, 64),                             # the first tokens see nothing
])
def test_few_rows_in_fp32(new, lens, hq, hk, d, path):
    import torch
    x = Batch(15, new, lens, hq, hk, d, 8, "fp32", path=path)
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    r_out, r_lse, e_out, e_lse = x.want()
    within(out, r_out, e_out, "out")
    within(lse, r_lse, e_lse, "lse")
    out2, lse2 = x.cache.attention(x.q)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0), ("fp32", 1)])
def test_more_new_tokens_than_the_most_are_reported_when_the_most_is_zero(dtype, path):
    import torch
    import paper_2503_21817_b200 as sk
    x = Batch(16, (1, 2), (9, 20), 4, 2, 64, 8, dtype, max_new=0, path=path)
    out, lse = torch.full_like(x.q, 7.0), torch.full((3, 4), 7.0, device="cuda")
    x.cache.attention(x.q, out=out, lse=lse)
    with pytest.raises(sk.SkipFFNError, match="site 64"):
        x.cache.poll()
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
def test_chunks_of_which_whole_tiles_see_nothing(dtype, path):
    import torch
    x = Batch(17, (600, 300, 40), (3, 0, 20), 8, 2, 64, 8, dtype, path=path)
    out, lse = x.cache.attention(x.q, out=torch.full_like(x.q, 7.0))
    x.cache.poll()
    r_out, r_lse, e_out, e_lse = x.want()
    within(out, r_out, e_out, "out")
    within(lse, r_lse, e_lse, "lse")
