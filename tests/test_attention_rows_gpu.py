"""Packed attention on the GPU: what one row's result may depend on.  Rows of other sequences that share a tile, and
keys whose scores are minus infinity, leave it as the definition has it."""
import numpy as np
import pytest

from gpu_util import to_host
from test_attention_gpu import _object, _tensors, _within, blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_finite_values_of_a_neighbour_do_not_reach_the_bits_of_a_sequence(dtype, path, causal):
    # the second sequence's first queries lie in the last row tile of the first one.  With queries along key 140 of
    # the first sequence their running maximum jumps in its second key block, by far more than 2^8: the first
    # sequence's rows in that tile must not notice.
    import torch
    lens, d = (150, 90), 64
    q, k, v, do, cu = _tensors(21, lens, 2, 2, d, dtype)
    a = _object(cu, 2, 2, d, dtype, causal, path=path)
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    wild = q.clone()
    wild[150:] = 100.0 * k[140]
    out2, lse2 = a.forward(wild, k, v)
    grads2 = a.backward(do, wild, k, v, out2, lse2)
    a.poll()
    for name, x, y in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads), (out2, lse2, *grads2)):
        assert torch.equal(x[:150], y[:150]), name


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("low", [-np.inf, -3e38])
@pytest.mark.parametrize("blind", [3, 64, 128, 200])
def test_keys_whose_scores_are_minus_infinity(dtype, path, low, blind):
    # the first `blind` keys score minus infinity for every query, as an infinite key or because the product leaves fp32:
    # their probability is zero, so rows that also see a later key have a finite answer (the last key block's, where
    # the first ones hold nothing), and rows that do not have none
    lens, d = (300,), 64
    q, k, v, do, cu = _tensors(22, lens, 4, 2, d, dtype)
    q[..., 0] = 1.0 if np.isinf(low) else 3e38
    k[:, :, 0] = 0.0
    k[:blind, :, 0] = low
    a = _object(cu, 4, 2, d, dtype, path=path)
    out, lse = a.forward(q, k, v)
    a.poll()
    Q, K, V = (to_host(t) for t in (q, k, v))
    Q[..., 0] = 0.0                                       # the answer without the blind keys
    K[..., 0] = 0.0
    worst = 0.0
    g, u = (d + 300 + 16) * 2.0 ** -24, blocks.HALF_STEP[dtype]
    for h in range(4):
        s = d ** -0.5 * Q[:, h] @ K[:, h // 2].T
        s = np.where(np.tril(np.ones_like(s, dtype=bool)), s, -np.inf)
        s[:, :blind] = -np.inf
        s = s[blind:]
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        r_lse = (top + np.log(p.sum(1, keepdims=True)))[:, 0]
        p /= p.sum(1, keepdims=True)
        es = g * (d ** -0.5 * np.abs(Q[blind:, h]) @ np.abs(K[:, h // 2]).T).max(1, keepdims=True)
        r_out = p @ V[:, h // 2]
        # the bounds of oracle/blocks.py for these rows
        e_out = (u + g + 2 * es + 2.0 ** -20) * (p @ np.abs(V[:, h // 2])) + u * np.abs(r_out)
        _within(out[blind:, h], r_out, e_out, f"out of head {h}")
        _within(lse[blind:, h], r_lse, es[:, 0] + g + 2.0 ** -22 * (1 + np.abs(r_lse)), f"lse of head {h}")
    assert not np.isfinite(to_host(lse[:blind])).any()


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 128), (3, 3, 40), (5, 1, 64), (64, 1, 32)])
def test_a_row_that_sees_one_key_has_no_gradient_of_its_score(dtype, path, causal, hq, hk, d):
    # P = 1 whatever the score: dq = 0, no contribution to dk, and dv gets dout as it is.  Exactly: what is left of
    # dP - delta when the two are summed in different orders is no gradient.
    import torch
    lens = (1, 1, 0, 1)
    q, k, v, do, cu = _tensors(23, lens, hq, hk, d, dtype)
    a = _object(cu, hq, hk, d, dtype, causal, path=path)
    out, lse = a.forward(q, k, v)
    dq, dk, dv = a.backward(do, q, k, v, out, lse)
    a.poll()
    assert torch.equal(out, v.repeat_interleave(hq // hk, 1))
    assert not dq.any() and not dk.any()
    want = to_host(do).reshape(3, hk, hq // hk, d)
    u = blocks.HALF_STEP[dtype]
    # the group's sum: at most 64 additions in fp32 of values whose P is 1 to (1 + |lse|) 2^-22; one rounding
    bound = (64 * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(to_host(lse)).max())) * np.abs(want).sum(2) + u * np.abs(want.sum(2))
    _within(dv, want.sum(2), bound, "dv")
    # a longer causal sequence: its first token
    if causal:
        q, k, v, do, cu = _tensors(24, (200, 33), hq, hk, d, dtype)
        a = _object(cu, hq, hk, d, dtype, causal, path=path)
        out, lse = a.forward(q, k, v)
        dq, dk, dv = a.backward(do, q, k, v, out, lse)
        assert not dq[0].any() and not dq[200].any() and bool(dq[1].any())
        # ... which adds nothing to dk: without its dout the same bits
        none = do.clone()
        none[0] = none[200] = 0
        assert torch.equal(dk, a.backward(none, q, k, v, out, lse)[1])


@pytest.mark.parametrize("dtype,path", [("bf16", 0), ("bf16", 1), ("fp32", 0)])
def test_a_gradient_that_is_not_finite_shows_where_a_row_sees_one_key(dtype, path):
    import torch
    q, k, v, do, cu = _tensors(25, (1, 40), 4, 2, 64, dtype)
    do[0, 0, 3] = float("nan")
    do[1, 0, 3] = float("inf")
    a = _object(cu, 4, 2, 64, dtype, path=path)
    out, lse = a.forward(q, k, v)
    dq, dk, dv = a.backward(do, q, k, v, out, lse)
    a.poll()
    for i in (0, 1):
        assert not torch.isfinite(dq[i, 0]).any() and not torch.isfinite(dk[i, 0]).any() and not torch.isfinite(dv[i, 0, 3])
        assert bool(torch.isfinite(dq[i, 2:]).all()) and bool(torch.isfinite(dk[:, 1]).all())
