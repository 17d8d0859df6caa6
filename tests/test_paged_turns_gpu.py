"""The paged cache's kernels where their loops over sequences, tiles and rows take more than one turn."""
import numpy as np
import pytest

from cache_util import Batch, normal, within
from gpu_util import to_host
from oracle import cache as oc
from test_paged_evict_gpu import _expect, _same_bits, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("kind", ["few", "more", "both"])
def test_thousands_of_sequences(kind, dtype, path):
    # 2500: ten turns of the walk of few rows, seven of the weights', three of the list, whose searches leave shared memory
    import torch
    n, hq, hk, d, page = 2500, 8, 1, 16, 8
    new = [{"few": i % 3, "more": 3 if i % 5 else 0, "both": (0, 1, 2, 3, 9)[i % 5]}[kind] for i in range(n)]
    lens = [max(m, 1 + 7 * i % 19) if i % 11 else 0 for i, m in enumerate(new)]
    new = [m if length else 0 for m, length in zip(new, lens)]
    x = Batch(41, new, lens, hq, hk, d, page, dtype, path=path)
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    r_out, r_lse, e_out, e_lse = x.want()
    within(out, r_out, e_out, "out")
    within(lse, r_lse, e_lse, "lse")
    width = max(lens)
    w = x.cache.weights(x.q, lse, width=width)
    x.cache.poll()
    r_w, e_w = oc.weights(to_host(x.q), x.keys, to_host(lse), x.cu, lens, hk, x.scale, width)
    within(w, r_w, e_w, "weights")


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("fp32", 0)])
def test_thousands_of_tiles(dtype, path):
    # 64 heads a kv head: a tile has 4 tokens in bf16, one in fp32; three sequences of 3000 tokens, the first of which see nothing
    new, lens, hq, hk, d = (3000, 3000, 2999), (40, 3000, 3100), 64, 1, 8
    x = Batch(42, new, lens, hq, hk, d, 64, dtype, path=path)
    out, lse = x.cache.attention(x.q)
    x.cache.poll()
    q = to_host(x.q)
    for s, (m, length) in enumerate(zip(new, lens)):
        for i in sorted({*range(0, m, 211), m - 1, m - 2, m - length if m > length else 0}):
            t, keys = x.cu[s] + i, max(0, length - m + i + 1)
            args = (q[t:t + 1], [x.keys[s][:keys]], [x.values[s][:keys]], [0, 1], [keys], x.scale, dtype)
            r_out, r_lse, e_out, e_lse = oc.attention(*args)
            within(out[t:t + 1], r_out, e_out, "out")
            within(lse[t:t + 1], r_lse, e_lse, "lse")


@pytest.mark.parametrize("lens,budget,sinks,recent,kind", [
    ((40001, 33000, 5), 5000, 4, 100, "spread"),            # a CTA's part is more than it holds in registers
    ((36000,), 35990, 0, 1, "ties"),                        # nearly all stay
    ((36000,), 1, 0, 0, "odd"),
    ((9001, 8200) + tuple(1 + 31 * i % 90 for i in range(298)), 700, 1, 9, "spread"),   # one CTA a pair
])
def test_eviction_of_more_rows_than_a_cluster_holds(lens, budget, sinks, recent, kind):
    import torch
    hk, d, page = 1, 8, 64
    x = Batch(43, [0] * len(lens), lens, hk, hk, d, page)
    w = _weights(7, len(lens), hk, max(lens), kind)
    kept, new = _expect(x, w, budget, sinks, recent)
    y = Batch(44, [0] * len(lens), new, hk, hk, d, page)
    rows = [[t[torch.from_numpy(x.table[s]).cuda().long()[torch.from_numpy(kept[s, 0, :m]).cuda().long() // page],
               torch.from_numpy(kept[s, 0, :m]).cuda().long() % page].clone() for t in (x.k, x.v)] for s, m in enumerate(new)]
    for into in (y.cache, None):
        got, got_lens, got_w = x.cache.evict(w, budget, sinks=sinks, recent=recent, into=into)
        x.cache.poll()
        assert np.array_equal(got.cpu().numpy(), kept) and got_lens.tolist() == new
        z = x if into is None else y
        for s, m in enumerate(new):
            j = torch.arange(m, device="cuda")
            p = z.d_table[s].long()[j // page]
            assert _same_bits(z.k[p, j % page], rows[s][0]) and _same_bits(z.v[p, j % page], rows[s][1])
            want = w.cpu().numpy()[s, 0, kept[s, 0, :m]]
            assert np.array_equal(got_w[s, 0, :m].cpu().numpy(), want, equal_nan=True) and not got_w[s, 0, m:].any()


def test_from_a_compacted_prompt_through_several_evictions():
    """The prompt's kept keys and values to pages, answers, weights that go on after an eviction."""
    import torch
    import paper_2503_21817_b200 as sk
    lens, hq, hk, d, page, budget, steps = (90, 160, 33), 8, 2, 64, 16, 40, 3
    n, n_seq = sum(lens), len(lens)
    cu = [0, 90, 250, 283]
    mask = (torch.rand(n, generator=torch.Generator().manual_seed(1)) < 0.5).to(torch.uint8)
    mask[[0, 90, 250]] = 0
    kv = torch.stack((normal(1, n, hk, d), normal(2, n, hk, d)))
    ctx = sk.SkipFFN(64, 64, n)
    ctx.plan(mask.cuda())
    pruned, kept_cu = ctx.kv_compact(kv, cu_seqlens=cu)
    cuts = kept_cu.tolist()
    held = [[to_host(kv)[i, a:b][mask[a:b].numpy() == 0] for i in range(2)] for a, b in zip(cu, cu[1:])]
    left = [h[0].shape[0] for h in held]
    assert cuts == [0, *np.cumsum(left).tolist()]
    x = Batch(45, left, [m + 2 * steps for m in left], hq, hk, d, page, max_new=max(left))
    x.k.fill_(float("nan")), x.v.fill_(float("nan"))
    x.d_cu.copy_(kept_cu), x.d_lens.copy_(kept_cu[1:] - kept_cu[:-1])
    x.cache.append(pruned[0], pruned[1])                         # rows behind the last kept one belong to no sequence
    x.cache.poll()
    x.d_cu.copy_(torch.arange(n_seq + 1, dtype=torch.int32))
    width = x.table.shape[1] * page
    gathered = torch.zeros(n_seq, hk, width, device="cuda")
    total = [np.zeros((hk, m)) for m in left]
    for step in range(2 * steps):
        x.d_lens.add_(1)
        q, k, v = normal(50 + step, n_seq, hq, d), normal(60 + step, n_seq, hk, d), normal(70 + step, n_seq, hk, d)
        x.cache.append(k, v)
        out, lse = x.cache.attention(q)
        gathered = x.cache.weights(q, lse, prior=gathered, out=gathered)
        x.cache.poll()
        for s in range(n_seq):
            held[s] = [np.concatenate((t, to_host(r[s:s + 1]))) for t, r in zip(held[s], (k, v))]
        now = [h[0].shape[0] for h in held]
        assert x.d_lens.tolist() == now
        r_out, r_lse, e_out, e_lse = oc.attention(to_host(q), [h[0] for h in held], [h[1] for h in held], [0, 1, 2, 3], now, d ** -0.5)
        within(out, r_out, e_out, "out")
        within(lse, r_lse, e_lse, "lse")
        prior = np.zeros((n_seq, hk, width))
        for s in range(n_seq):
            prior[s, :, :total[s].shape[1]] = total[s]
        r_w, e_w = oc.weights(to_host(q), [h[0] for h in held], to_host(lse), [0, 1, 2, 3], now, hk, d ** -0.5, width, prior)
        within(gathered, r_w, e_w, "weights")
        total = [to_host(gathered)[s, :, :m] for s, m in enumerate(now)]
        if step % steps == steps - 1:
            kept, new, rest = x.cache.evict(gathered, budget, sinks=1, recent=4)
            x.cache.poll()
            rows = kept.cpu().numpy()
            for s in range(n_seq):
                m = min(now[s], budget)
                held[s] = [np.stack([t[rows[s, h, :m], h] for h in range(hk)], 1) for t in held[s]]
                total[s] = to_host(rest)[s, :, :m]
            x.d_lens.copy_(new)
            # wide enough for the rows to come: the returned weights end with the rows kept
            gathered = torch.zeros(n_seq, hk, width, device="cuda")
            gathered[..., :budget] = rest
