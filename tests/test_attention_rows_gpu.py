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
