"""fp64 statements of rotary positions, attention over a paged cache, the weights of its rows and eviction, with elementwise
error bounds (numpy; test infrastructure).  Written from the formulas, one sequence and one head at a time.

Bounds.  `u` is the relative half step of the results' type, `g` the relative error of a fp32 sum of that many terms in any
order.  A computed cosine or sine is off by at most TRIG: half a step of the reduced angle (below pi / 4), two of the
function, the angle's last bit; and |t| 2^-52 because frequency and product are 64-bit numbers."""
from __future__ import annotations

import numpy as np

from .blocks import HALF_STEP

TRIG = 6 * 2.0 ** -24
SUM = 64 * 2.0 ** -24       # a row's sum of squares or products (at most 16 in a thread, 5 shuffles) and what is done with it


def pairs_of(d, rot, interleaved):
    """Columns (a, b) of every rotated pair."""
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)


def angles(pos, freq, axis):
    """[tokens, pairs] from positions [axes, tokens]."""
    return np.asarray(pos, dtype=np.float64)[np.asarray(axis, dtype=int)].T * np.asarray(freq, dtype=np.float64)


def _turn(x, t, a, b, sign):
    """Rotated x [tokens, heads, d] and the bound of its error."""
    y, e = x.copy(), np.zeros_like(x)
    c, s = np.cos(t)[:, None], sign * np.sin(t)[:, None]
    xa, xb = x[..., a], x[..., b]
    y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
    e[..., a] = e[..., b] = (np.abs(xa) + np.abs(xb)) * (TRIG + np.abs(t)[:, None] * 2.0 ** -52)
    return y, e


def rotary_forward(x, pos, freq, axis, rot, interleaved=False, gamma=None, eps=1e-6, dtype="bf16"):
    """``(y, bound)`` for x [tokens, heads, d]."""
    u, (a, b) = HALF_STEP[dtype], pairs_of(x.shape[-1], rot, interleaved)
    n = x if gamma is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gamma
    t = angles(pos, freq, axis) if rot else np.zeros((x.shape[0], 0))
    y, e = _turn(n, t, a, b, 1.0)
    # columns that are not turned have the norm's error alone
    en = np.zeros_like(x) if gamma is None else SUM * np.abs(n)
    e[..., a] += en[..., a] + en[..., b]
    e[..., b] = e[..., a]
    rest = np.setdiff1d(np.arange(x.shape[-1]), np.concatenate((a, b)))
    e[..., rest] = en[..., rest]
    return y, e + u * np.abs(y)


def rotary_backward(dy, x, pos, freq, axis, rot, interleaved=False, gamma=None, eps=1e-6, dtype="bf16", dw_dtype=None):
    """``((dx, dgamma), bounds)``; dgamma is None without gamma."""
    u, uw, (a, b) = HALF_STEP[dtype], HALF_STEP[dw_dtype or dtype], pairs_of(x.shape[-1], rot, interleaved)
    t = angles(pos, freq, axis) if rot else np.zeros((x.shape[0], 0))
    dn, e = _turn(dy, t, a, b, -1.0)
    if gamma is None:
        return (dn, None), (e + u * np.abs(dn), None)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    w = dn * gamma
    m = (w * x).mean(-1, keepdims=True)
    dx = r * (w - x * r * r * m)
    edx = (r * np.abs(gamma) * e + r ** 3 * np.abs(x) * (np.abs(gamma) * e * np.abs(x)).mean(-1, keepdims=True)
           + SUM * (r * np.abs(w) + 3 * r ** 3 * np.abs(x) * np.abs(w * x).mean(-1, keepdims=True)) + u * np.abs(dx))
    dg = (dn * x * r).sum((0, 1))
    rows = x.shape[0] * x.shape[1]
    edg = (e * np.abs(x) * r).sum((0, 1)) + (rows * 2.0 ** -24 + SUM) * np.abs(dn * x * r).sum((0, 1)) + uw * np.abs(dg)
    return (dx, dg), (edx, edg)


def rows_of(pages, table, length):
    """Rows 0 .. length - 1 of a sequence: [length, heads, d] of pages [pages, page, heads, d]."""
    j = np.arange(length)
    page = pages.shape[1]
    return pages[np.asarray(table)[j // page], j % page]


def _scores(q, k, scale, off):
    """(scores with minus infinity where a row is not seen, bound of their error) of one head; q [n, d], k [len, d]."""
    s = scale * (q @ k.T)
    seen = np.arange(k.shape[0])[None, :] <= off + np.arange(q.shape[0])[:, None]
    g = (q.shape[1] + 16) * 2.0 ** -24
    return np.where(seen, s, -np.inf), g * scale * (np.abs(q) @ np.abs(k).T)


def attention(q, keys, values, cu, lens, scale, dtype="bf16"):
    """``(out, lse, bound_out, bound_lse)``: q [N, Hq, d]; keys / values: a list with [len, Hk, d] for each sequence."""
    n, hq, d = q.shape
    u = HALF_STEP[dtype]
    out, eo = np.zeros_like(q), np.zeros_like(q)
    lse, el = np.full((n, hq), -np.inf), np.zeros((n, hq))
    for s, length in enumerate(lens):
        a, b = cu[s], cu[s + 1]
        for h in range(hq if b > a and length else 0):
            k, v = (t[s][:, h * t[s].shape[1] // hq] for t in (keys, values))
            z, ez = _scores(q[a:b, h], k, scale, length - (b - a))
            top = z.max(1, keepdims=True)
            live = top[:, 0] > -np.inf
            p = np.exp(z - np.where(live[:, None], top, 0.0))
            den = p.sum(1, keepdims=True)
            p /= np.where(live[:, None], den, 1.0)
            ds = np.where(np.isfinite(z), ez, 0.0).max(1, keepdims=True)
            g = (length + 64) * 2.0 ** -24
            out[a:b, h] = p @ v
            eo[a:b, h] = (u + g + 2 * ds + 2.0 ** -20) * (p @ np.abs(v)) + u * np.abs(out[a:b, h])
            lse[a:b, h] = np.where(live, (top + np.log(np.where(live[:, None], den, 1.0)))[:, 0], -np.inf)
            el[a:b, h] = ds[:, 0] + g + 2.0 ** -22 * (1.0 + np.where(live, np.abs(lse[a:b, h]), 0.0))
    return out, lse, eo, el


def weights(q, keys, lse, cu, lens, heads_kv, scale, width, prior=None):
    """``(weights [n_seq, heads_kv, width], bound)`` for the given lse."""
    hq = q.shape[1]
    w, e = np.zeros((len(lens), heads_kv, width)), np.zeros((len(lens), heads_kv, width))
    for s, length in enumerate(lens):
        a, b = cu[s], cu[s + 1]
        if prior is not None:
            w[s, :, :length] = prior[s, :, :length]
        for h in range(hq if b > a else 0):
            z, ez = _scores(q[a:b, h], keys[s][:, h * heads_kv // hq], scale, length - (b - a))
            l = lse[a:b, h][:, None]
            x = np.where(l > -np.inf, z - np.where(l > -np.inf, l, 0.0), -np.inf)
            p = np.exp(x)
            w[s, h * heads_kv // hq, :length] += p.sum(0)
            # exponent: error of the score and of the difference; 2 steps of the exponential; the sum over rows
            rel = np.where(np.isfinite(x), ez + 2.0 ** -22 * (1.0 + np.abs(x)), 0.0)
            e[s, h * heads_kv // hq, :length] += (p * (rel + 2.0 ** -22 + ((b - a) * hq + 16) * 2.0 ** -24)).sum(0)
    return w, e + 2.0 ** -23 * np.abs(w)


def evict(w, length, budget, sinks, recent):
    """Rows of one sequence and head that stay, ascending; w [>= length] fp32."""
    if length <= budget:
        return list(range(length))
    free = [j for j in range(sinks, length - recent)]
    # largest first, NaN last, lower row first among equals
    free.sort(key=lambda j: (bool(np.isnan(w[j])), 0.0 if np.isnan(w[j]) else -float(w[j]), j))
    keep = list(range(sinks)) + free[:budget - sinks - recent] + list(range(length - recent, length))
    return sorted(keep)
