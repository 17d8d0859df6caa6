"""Packed attention on the GPU against its fp64 statement: every element within the bound of the arithmetic
(oracle/blocks.py), at the sizes, groups, strides and neighbours where the kernels can go wrong."""
import math

import numpy as np
import pytest

from oracle import blocks
from gpu_util import to_host

pytestmark = pytest.mark.gpu


def _tensors(seed, lens, hq, hk, d, dtype, pad=0, fused=False):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n = sum(lens) + pad
    q, k, v, do = (torch.randn(n, h, d, generator=g).to(dt).cuda() for h in (hq, hk, hk, hq))
    if fused:
        q, k, v = torch.cat((q, k, v), 1).split((hq, hk, hk), 1)
    return q, k, v, do, [0] + [int(c) for c in np.cumsum(lens)]


def _object(cu, hq, hk, d, dtype, causal=True, **kw):
    import paper_2503_21817_b200 as sk
    return sk.PackedAttention(cu, hq, hk, d, dtype=sk.BF16 if dtype == "bf16" else sk.FP32, causal=causal, **kw)


def _within(got, want, bound, what):
    got = to_host(got)
    assert np.isfinite(got).all(), f"{what}: non-finite values"
    worst = np.max(np.abs(got - want) / np.maximum(bound, 1e-300)) if got.size else 0.0
    assert worst <= 1.0, f"{what}: an element is {worst:.3f} times its bound away"


def _check(a, q, k, v, do, cu, scale, causal, dtype):
    import torch
    n = cu[-1]
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    a.poll()
    Q, K, V, G = (to_host(t)[:n] for t in (q, k, v, do))
    r_out, r_lse, e_out, e_lse = blocks.attention_forward(Q, K, V, cu, scale, causal, dtype)
    _within(out[:n], r_out, e_out, "out")
    _within(lse[:n], r_lse, e_lse, "lse")
    refs, errs = blocks.attention_backward(Q, K, V, G, cu, scale, causal, dtype)
    for name, got, r, e in zip(("dq", "dk", "dv"), grads, refs, errs):
        _within(got[:n], r, e, name)
    # fixed order of every sum: the same bits again
    out2, lse2 = a.forward(q, k, v)
    again = a.backward(do, q, k, v, out2, lse2)
    for x, y in zip((out, lse, *grads), (out2, lse2, *again)):
        assert torch.equal(x[:n], y[:n])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,hq,hk,d,causal", [
    ((1,), 4, 1, 128, True),                       # one token
    ((1, 2, 0, 1), 2, 2, 64, True),                # single tokens, an empty sequence
    ((15, 16, 17), 8, 2, 128, True),               # around the 16-row MMA step
    ((127, 128, 129), 2, 2, 64, True),             # around a tile, one head per tile
    ((255, 256, 257), 1, 1, 128, False),
    ((32, 64, 65, 31), 8, 2, 128, True),           # around the 32 tokens of a tile of 4 heads
    ((577, 40), 4, 4, 64, False),                  # vision tower
    ((616, 133), 8, 2, 128, True),                 # decoder
    ((300, 7), 10, 2, 96, True),                   # groups of 5: 125 of 128 rows, 96 columns
    ((260,), 7, 1, 80, True),                      # group of 7
    ((130, 70), 12, 4, 40, False),                 # group of 3, 40 columns
    ((70, 200), 64, 1, 32, True),                  # 64 heads share one: two tokens per tile
    ((90,), 3, 3, 8, True),                        # the narrowest head
])
def test_against_64_bits(lens, hq, hk, d, causal, dtype):
    q, k, v, do, cu = _tensors(sum(lens) + hq, lens, hq, hk, d, dtype)
    _check(_object(cu, hq, hk, d, dtype, causal), q, k, v, do, cu, d ** -0.5, causal, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores_other_scale_and_fused_strides(dtype):
    # scores up to some hundreds: the running maximum moves block by block, the sums must follow
    q, k, v, do, cu = _tensors(5, (400, 129), 8, 2, 64, dtype, fused=True)
    for scale in (2.0, 0.01):
        _check(_object(cu, 8, 2, 64, dtype, scale=scale), q, k, v, do, cu, scale, True, dtype)


def test_plain_fma_path_agrees_in_bf16():
    import paper_2503_21817_b200 as sk
    q, k, v, do, cu = _tensors(6, (200, 33), 8, 2, 128, "bf16")
    _check(_object(cu, 8, 2, 128, "bf16", path=sk.PATH_SIMT), q, k, v, do, cu, 128 ** -0.5, True, "bf16")


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_neighbours_and_rows_behind_the_batch_do_not_reach_a_sequence(dtype, path, causal):
    import torch
    lens, pad = (37, 150, 61), 9
    q, k, v, do, cu = _tensors(7, lens, 4, 2, 64, dtype, pad=pad)
    a = _object(cu, 4, 2, 64, dtype, causal, path=path)
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    lo, hi, n = cu[1], cu[2], cu[3]
    bad = [t.clone() for t in (q, k, v, do)]
    for t, x in zip(bad, (float("nan"), float("inf"), -float("inf"), float("nan"))):
        t[:lo] = x
        t[hi:] = x
    mark = lambda t: torch.full_like(t, 7.0)
    out2, lse2 = a.forward(*bad[:3], out=mark(out), lse=mark(lse))
    grads2 = a.backward(bad[3], *bad[:3], out2, lse2, *(mark(g) for g in grads))
    a.poll()
    for x, y in zip((out, lse, *grads), (out2, lse2, *grads2)):
        assert torch.equal(x[lo:hi], y[lo:hi])
        assert bool((y[n:] == 7.0).all())                      # rows behind the last sequence are left alone


def test_long_sequence_rows_against_64_bits():
    # 9001 keys, sampled rows: the first, the last, and around tile seams
    import torch
    q, k, v, _, cu = _tensors(8, (9001,), 2, 1, 128, "bf16")
    out, lse = _object(cu, 2, 1, 128, "bf16").forward(q, k, v)
    Q, K, V = (to_host(t) for t in (q, k, v))
    for i in (0, 63, 64, 127, 128, 4095, 4096, 8191, 8999, 9000):
        r_out, r_lse, e_out, e_lse = blocks.attention_forward(Q[i:i + 1], K[:i + 1], V[:i + 1], [0, 1], 128 ** -0.5, False, "bf16") \
            if i == 0 else _row(Q[i], K[:i + 1], V[:i + 1])
        _within(out[i:i + 1], r_out, e_out, f"row {i}")
        _within(lse[i:i + 1], r_lse, e_lse, f"lse {i}")


def _row(q, K, V):
    """One query against all keys, as the last row of a sequence."""
    n, d = K.shape[0], K.shape[2]
    s = d ** -0.5 * np.einsum("hd,nd->hn", q, K[:, 0])
    top = s.max(1, keepdims=True)
    p = np.exp(s - top)
    den = p.sum(1, keepdims=True)
    p /= den
    g, u = (n + d + 16) * 2.0 ** -24, 2.0 ** -8
    es = g * (d ** -0.5 * np.einsum("hd,nd->hn", np.abs(q), np.abs(K[:, 0]))).max(1, keepdims=True)
    out, lse = p @ V[:, 0], (top + np.log(den))[:, 0]
    e = (u + g + 2 * es + 2.0 ** -20) * (p @ np.abs(V[:, 0])) + u * np.abs(out)
    return out[None], lse[None], e[None], (es[:, 0] + g + 2.0 ** -22 * (1 + np.abs(lse)))[None]


def test_gradient_against_differences():
    # fp32 kernels against central differences of the 64-bit forward.  The difference is exact to
    # h^2 f''' / 6 + 2^-52 |f| / h ~ 1e-8 here; the kernels' sums err by less than 2e-5 of their absolute terms.
    import torch
    q, k, v, do, cu = _tensors(9, (40, 70), 4, 2, 64, "fp32")
    a = _object(cu, 4, 2, 64, "fp32")
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    host = [to_host(t) for t in (q, k, v)]
    G, r = to_host(do), np.random.default_rng(0)
    f = lambda *t: float(np.sum(G * blocks.attention_forward(*t, cu, 0.125, True, "fp32")[0]))
    for i in range(3):
        e = r.standard_normal(host[i].shape)
        moved = lambda s: [t + s * e if j == i else t for j, t in enumerate(host)]
        num = (f(*moved(1e-4)) - f(*moved(-1e-4))) / 2e-4
        got = to_host(grads[i])
        assert abs(num - np.sum(got * e)) <= 2e-5 * np.abs(got * e).sum() + 1e-6


def test_fused_gradients_other_stream_capture_and_replay():
    import torch
    lens, hq, hk, d = (100, 257), 8, 2, 128
    q, k, v, do, cu = _tensors(10, lens, hq, hk, d, "bf16", fused=True)
    a = _object(cu, hq, hk, d, "bf16")
    out, lse = a.forward(q, k, v)
    ref = a.backward(do, q, k, v, out, lse)
    n = cu[-1]
    grad = torch.full((n, hq + 2 * hk, d), 3.0, dtype=torch.bfloat16, device="cuda")
    views = grad.split((hq, hk, hk), 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out2, lse2 = a.forward(q, k, v)
        a.backward(do, q, k, v, out2, lse2, *views)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, out2) and all(torch.equal(x, y) for x, y in zip(ref, views))
    # two captured graphs of one object, replayed in turn on new inputs
    graphs = []
    for seed in (11, 12):
        t = _tensors(seed, lens, hq, hk, d, "bf16", fused=True)[:4]
        want = (*(r := a.forward(*t[:3])), *a.backward(t[3], *t[:3], *r))
        held = [x.clone() for x in t]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, l = a.forward(*held[:3])
            got = (o, l, *a.backward(held[3], *held[:3], o, l))
        graphs.append((graph, got, want, held))          # the graph reads `held` at every replay
    for _ in range(2):
        for graph, got, *_ in graphs:
            for x in got:
                x.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _g, got, want, _h in graphs:
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    a.poll()


@pytest.mark.parametrize("path", [0, 1])
def test_offsets_past_32_bits(path):
    # tokens 2^21 elements apart: the last ones lie behind 2^31 elements.  Same bits as from packed arrays.
    import torch
    q, k, v, do, cu = _tensors(15, (700, 400), 4, 2, 64, "bf16")
    a = _object(cu, 4, 2, 64, "bf16", path=path)
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    far = torch.empty(1100, 1 << 21, dtype=torch.bfloat16, device="cuda")
    places = iter(range(0, 1 << 21, 256))
    def moved(t):
        x = next(places)
        w = far[:, x:x + t.shape[1] * t.shape[2]].view(1100, t.shape[1], t.shape[2])
        return w.copy_(t)
    Q, K, V, G = (moved(t) for t in (q, k, v, do))
    O, dQ, dK, dV = (moved(torch.zeros_like(t)) for t in (q, q, k, v))
    O, L = a.forward(Q, K, V, out=O)
    a.backward(G, Q, K, V, O, L, dQ, dK, dV)
    a.poll()
    assert torch.equal(L, lse) and all(torch.equal(x, y) for x, y in zip((O, dQ, dK, dV), (out, *grads)))


def test_work_lists_outlive_calls_on_another_stream():
    # the object is dropped while a call on a side stream has not run yet: its lists may not be handed out again
    import torch
    q, k, v, do, cu = _tensors(14, (64,) * 40, 4, 2, 64, "bf16")
    a = _object(cu, 4, 2, 64, "bf16")
    want, _ = a.forward(q, k, v)
    address, size = a._plan.data_ptr(), a._plan.numel()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)                         # about half a second
        got, _ = a.forward(q, k, v)
        done = side.record_event()
    del a
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(8)]
    pending = not done.query()                                   # a call that has ended no longer needs the lists
    assert not pending or all(t.data_ptr() != address for t in others)
    side.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    import torch
    import paper_2503_21817_b200 as sk
    q, k, v, do, cu = _tensors(13, (20,), 4, 2, 64, "bf16")
    a = _object(cu, 4, 2, 64, "bf16")
    out, lse = a.forward(q, k, v)
    for bad in ((q.float(), k, v), (q[:10], k, v), (q, k[:, :1], v), (q.transpose(0, 1), k, v), (q.cpu(), k, v),
                (q, k, v[..., :32]), (q.view(20, -1), k, v)):
        with pytest.raises(ValueError):
            a.forward(*bad)
    with pytest.raises(ValueError):
        a.forward(q, k, v, lse=lse.double())
    wide = torch.zeros(20, 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[:, :256].view(20, 4, 64)    # 8-byte stride
    for bad in ((wide, k, v), (q[1:], k, v)):
        with pytest.raises((sk.SkipFFNError, ValueError)):
            a.forward(*bad)
    with pytest.raises(sk.SkipFFNError):
        a.forward(q, k, v, out=q)
    for spread in (do[:1].expand(20, 4, 64), do[:, :1].expand(20, 4, 64), do[..., :1].expand(20, 4, 64)):     # gradients of sums
        with pytest.raises((sk.SkipFFNError, ValueError)):
            a.backward(spread, q, k, v, out, lse)
    for kw in (dict(dq=q), dict(dk=v), dict(dv=k), dict(dk=v.clone(), dv=None, dq=out)):
        with pytest.raises(sk.SkipFFNError):
            a.backward(do, q, k, v, out, lse, **kw)
    # results on top of the statistics, at the C entry: dq, dk, dv on lse; scratch on any of the nine arrays
    big = torch.empty(20, 4, 64, dtype=torch.bfloat16, device="cuda")
    rows = [do, q, k, v, out, lse, big, torch.empty_like(k), torch.empty_like(k), torch.empty(a.scratch_bytes, dtype=torch.uint8, device="cuda")]
    def at_c(i, p):
        p = [t.data_ptr() if j != i else p for j, t in enumerate(rows)]
        ld = [256, 256, 128, 128, 256, None, 256, 128, 128, None]
        flat = [x for y, z in zip(p, ld) for x in ((y,) if z is None else (y, z))]
        return a.lib.skipffn_attention_backward(a._handle, *flat, a.scratch_bytes, None)
    assert [at_c(i, lse.data_ptr()) for i in (6, 7, 8)] == [1] * 3
    assert [at_c(9, t.data_ptr()) for t in rows[:9]] == [1] * 9
    assert at_c(9, rows[9].data_ptr() + 8) == 1
    same = torch.empty_like(k)
    with pytest.raises(sk.SkipFFNError):
        a.backward(do, q, k, v, out, lse, dk=same, dv=same)
    for bad in (([0, 5, 3], 4, 2, 64), ([1, 5], 4, 2, 64), ([0, 5], 4, 3, 64), ([0, 5], 4, 2, 60), ([0, 5], 4, 2, 136), ([], 4, 2, 64)):
        with pytest.raises(sk.SkipFFNError):
            sk.PackedAttention(*bad)
    with pytest.raises(ValueError):
        sk.PackedAttention([0, 1 << 31], 4, 2, 64)
    # a stride that would leave 64 bits, and one that is no multiple of 16 bytes, at the C entry
    f, p = a.lib.skipffn_attention_forward, (q.data_ptr(), k.data_ptr(), v.data_ptr(), torch.empty_like(q).data_ptr(), lse.data_ptr())
    call = lambda ld: f(a._handle, p[0], ld, p[1], 128, p[2], 128, p[3], 256, torch.empty_like(lse).data_ptr(), None)
    assert [call(ld) for ld in (1 << 62, 1 << 40, -256, 0, 252, 248)] == [1] * 6
    # an empty batch is a batch
    e = sk.PackedAttention([0, 0], 4, 2, 64)
    o, l = e.forward(q[:0], k[:0], v[:0])
    assert o.shape == (0, 4, 64) and l.shape == (0, 4)
    assert [t.shape[0] for t in e.backward(do[:0], q[:0], k[:0], v[:0], o, l)] == [0, 0, 0]
    e.poll()
