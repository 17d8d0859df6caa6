"""fp64 statements of packed attention and layer normalisation, with elementwise error bounds (numpy; test
infrastructure).  Written from the formulas, one sequence and one head at a time.

attention:  s_ij = scale q_i . k_j;  p_i = softmax_j s_ij over j <= i (causal) or all j of the sequence;
            out_i = sum_j p_ij v_j;  lse_i = log sum_j exp s_ij
            dv_j = sum_i p_ij do_i;  ds_ij = p_ij (do_i . v_j - do_i . out_i);
            dq_i = scale sum_j ds_ij k_j;  dk_j = scale sum_i ds_ij q_i   (i over all heads of the group)
layernorm:  y = (x - mean) rstd gamma + beta and its vjp.

Bounds.  `u` is the relative half step of the operands the second products and the results are rounded to
(2^-8 for bf16, 2^-24 for fp32) and `g` the relative error of a fp32 sum of that many terms in any order.
  out: every p_ij is rounded (u) and the result is rounded (u):   (u + g) sum_j p_ij |v_j| + u |out|
  lse: error of a score, g sum_d |q k| scale, plus rounding of the logarithm's result
  dv :                                         (u + g) sum_i p_ij |do_i| + u |dv|
  ds : relative u + g, plus p_ij times the error of delta_i = do_i . out_i, whose `out` carries its own
       bound;  dq, dk: sums of those against |k|, |q|, plus the rounding of the result."""
from __future__ import annotations

import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def _sequences(cu):
    return [(int(a), int(b)) for a, b in zip(cu, cu[1:]) if b > a]


def _probabilities(q, k, scale, causal):
    """(p, lse, bound of the error of a fp32 score) of one head of one sequence."""
    s = scale * (q @ k.T)
    if causal:
        s = np.where(np.tril(np.ones_like(s, dtype=bool)), s, -np.inf)
    top = s.max(axis=1, keepdims=True)
    e = np.exp(s - top)
    den = e.sum(axis=1, keepdims=True)
    es = scale * (np.abs(q) @ np.abs(k).T)
    return e / den, (top + np.log(den))[:, 0], np.where(np.isfinite(s), es, 0.0)


def attention_forward(q, k, v, cu, scale, causal, dtype="bf16"):
    """``(out, lse, bound_out, bound_lse)``; q [N, Hq, d], k / v [N, Hk, d] float64."""
    n, hq, d = q.shape
    group, u = hq // k.shape[1], HALF_STEP[dtype]
    out, eout = np.zeros_like(q), np.zeros_like(q)
    lse, else_ = np.zeros((n, hq)), np.zeros((n, hq))
    for a, b in _sequences(cu):
        g = (d + b - a + 16) * 2.0 ** -24
        for h in range(hq):
            kk, vv = k[a:b, h // group], v[a:b, h // group]
            p, l, es = _probabilities(q[a:b, h], kk, scale, causal)
            ds = g * es.max(axis=1, keepdims=True)              # error of the exponents
            out[a:b, h] = p @ vv
            eout[a:b, h] = (u + g + 2 * ds + 2.0 ** -20) * (p @ np.abs(vv)) + u * np.abs(out[a:b, h])
            lse[a:b, h] = l
            else_[a:b, h] = ds[:, 0] + g + 2.0 ** -22 * (1.0 + np.abs(l))
    return out, lse, eout, else_


def attention_backward(q, k, v, dout, cu, scale, causal, dtype="bf16", bound_out=None):
    """``((dq, dk, dv), (bounds))`` for upstream gradient ``dout``; ``bound_out``: error of the `out` that delta is
    formed from (default: the forward's bound)."""
    hq, d = q.shape[1:]
    group, u = hq // k.shape[1], HALF_STEP[dtype]
    if bound_out is None:
        bound_out = attention_forward(q, k, v, cu, scale, causal, dtype)[2]
    res = [np.zeros_like(t) for t in (q, k, v)]
    err = [np.zeros_like(t) for t in (q, k, v)]
    for a, b in _sequences(cu):
        g = (d + (b - a) * group + 16) * 2.0 ** -24
        for h in range(hq):
            hk = h // group
            Q, K, V, G = q[a:b, h], k[a:b, hk], v[a:b, hk], dout[a:b, h]
            p, l, es = _probabilities(Q, K, scale, causal)
            rel = g * es.max() + 2.0 ** -20 + 2.0 ** -22 * (1.0 + np.abs(l).max())    # relative error of p
            dp = G @ V.T
            delta = np.sum(p * dp, axis=1, keepdims=True)
            ds = p * (dp - delta)
            eds = (u + 2 * g + 2 * rel) * np.abs(ds) + p * (
                g * (np.abs(G) @ np.abs(V).T) + np.sum(np.abs(G) * bound_out[a:b, h], axis=1, keepdims=True)
                + g * np.sum(np.abs(G) * (p @ np.abs(V)), axis=1, keepdims=True))
            res[0][a:b, h] = scale * (ds @ K)
            err[0][a:b, h] = scale * ((eds + g * np.abs(ds)) @ np.abs(K)) + u * np.abs(res[0][a:b, h])
            res[1][a:b, hk] += scale * (ds.T @ Q)
            err[1][a:b, hk] += scale * ((eds + g * np.abs(ds)).T @ np.abs(Q))
            res[2][a:b, hk] += p.T @ G
            err[2][a:b, hk] += (u + g + 2 * rel) * (p.T @ np.abs(G))
    for i in (1, 2):
        err[i] += u * np.abs(res[i])
    return tuple(res), tuple(err)


def _bf16(x):
    """Nearest bf16 value of each finite entry (ties to even), as float64."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((b + (0x7fff + ((b >> 16) & 1))) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)


def attention_rounded(q, k, v, dout, cu, scale, causal, mistake=None):
    """``(out, dq, dk, dv)`` in fp64 but for the roundings to bf16 that the tensor-core kernels document: P as operand
    of out and dV, dS as operand of dK (in dQ it is the sum of two bf16 numbers: no rounding), delta from the rounded
    out, put right by the row sums of dS before dK is formed (rows of a tile whose keys are one block of 128: the exact
    delta), and each result.  Gives the size of error to expect.
    `mistake` plants one: "dropped" / "negated" correction of delta, "one number": dS rounded in dQ too."""
    hq, group = q.shape[1], q.shape[1] // k.shape[1]
    tokens = 128 // group                        # of a row tile
    out, dq, dk, dv = (np.zeros_like(t) for t in (q, q, k, v))
    correct = {"dropped": 0.0, "negated": -1.0}.get(mistake, 1.0)
    for a, b in _sequences(cu):
        for h in range(hq):
            hk = h // group
            Q, K, V, G = q[a:b, h], k[a:b, hk], v[a:b, hk], dout[a:b, h]
            p, _, _ = _probabilities(Q, K, scale, causal)
            P, dp = _bf16(p), G @ V.T
            out[a:b, h] = _bf16(P @ V)
            tile_end = np.minimum((np.arange(b - a) // tokens + 1) * tokens, b - a) if causal else np.full(b - a, b - a)
            delta = np.where(tile_end <= 128, np.sum(p * dp, axis=1), np.sum(G * out[a:b, h], axis=1))[:, None]
            ds = p * (dp - delta)
            dq[a:b, h] = scale * ((_bf16(ds) if mistake == "one number" else ds) @ K)
            delta = delta + correct * ds.sum(axis=1, keepdims=True)
            dk[a:b, hk] += scale * (_bf16(p * (dp - delta)).T @ Q)
            dv[a:b, hk] += P.T @ G
    return out, _bf16(dq), _bf16(dk), _bf16(dv)


# A fp32 sum of C values: at most 40 additions one after the other in a thread, ten shuffle or shared-memory
# levels of at most 32 more; 128 roundings bound every path, and the products around it.
_G = 128 * 2.0 ** -24


def layernorm_forward(x, gamma, beta, eps, dtype="bf16"):
    """``(y, mean, rstd, bound_y, bound_mean, bound_rstd)``; x [n, C] float64."""
    u = HALF_STEP[dtype]
    mean = x.mean(axis=1)
    z = x - mean[:, None]
    var = (z * z).mean(axis=1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = z * rstd[:, None] * gamma + beta
    emean = _G * np.abs(x).mean(axis=1)
    # var of values shifted by emean: second order in emean; each z carries emean and a rounding of |x|
    evar = _G * var + 2 * np.sqrt(var) * (emean + 2.0 ** -24 * np.abs(x).max(axis=1)) + (emean + 2.0 ** -24 * np.abs(x).max(axis=1)) ** 2
    erstd = rstd * (0.5 * evar / (var + eps) + _G)
    ey = (np.abs(gamma) * (rstd[:, None] * (emean[:, None] + 2.0 ** -24 * np.abs(x)) + np.abs(z) * erstd[:, None])
          + _G * (np.abs(y) + np.abs(beta)) + u * np.abs(y))
    return y, mean, rstd, ey, emean, erstd


def layernorm_backward(dy, x, gamma, mean, rstd, dtype="bf16", dw_dtype=None):
    """``((dx, dgamma, dbeta), bounds)`` from the given statistics."""
    u, n = HALF_STEP[dtype], x.shape[0]
    uw = HALF_STEP[dw_dtype or dtype]
    xh = (x - mean[:, None]) * rstd[:, None]
    exh = rstd[:, None] * 2.0 ** -23 * (np.abs(x) + np.abs(mean)[:, None]) + 2.0 ** -23 * np.abs(xh)
    t = dy * gamma
    m0, m1 = t.mean(axis=1, keepdims=True), (t * xh).mean(axis=1, keepdims=True)
    dx = rstd[:, None] * (t - m0 - xh * m1)
    em0 = _G * np.abs(t).mean(axis=1, keepdims=True)
    em1 = (_G * np.abs(t * xh) + np.abs(t) * exh).mean(axis=1, keepdims=True)
    edx = rstd[:, None] * (em0 + np.abs(xh) * em1 + exh * np.abs(m1) + 2.0 ** -22 * (np.abs(t) + np.abs(m0) + np.abs(xh * m1))) + u * np.abs(dx)
    g = (n + 256) * 2.0 ** -24
    dgamma, dbeta = (dy * xh).sum(axis=0), dy.sum(axis=0)
    edg = g * np.abs(dy * xh).sum(axis=0) + (np.abs(dy) * exh).sum(axis=0) + uw * np.abs(dgamma)
    edb = g * np.abs(dy).sum(axis=0) + uw * np.abs(dbeta)
    return (dx, dgamma, dbeta), (edx, edg, edb)
