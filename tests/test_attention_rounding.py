"""Relative Frobenius errors of packed attention: no larger than the roundings that the kernels document make them.  The
elementwise bounds of the other tests cover the worst case of every term at once; a lost correction of delta or a lost
half of dS stays far inside those, and outside these."""
import numpy as np
import pytest

from oracle import blocks

# sequences of more than one key block (shorter ones have the exact delta), scores large enough for delta to matter
CASES = [((300, 180), 8, 2, 128, 0.3, True), ((616, 133), 8, 2, 128, 0.3, True), ((255, 256, 257), 2, 2, 64, 0.3, False),
         ((300, 7), 10, 2, 96, 0.3, True), ((170, 200), 64, 1, 32, 0.6, True)]
# The limit is 1.04 times the error of oracle.blocks.attention_rounded on the same inputs.  It rounds the same quantities
# at the same places; the kernels round P before it is normalised, another draw of as many rounding errors.  The
# smallest result here has 11840 entries, the sampling error of its root mean square is 1 / sqrt(2 x 11840) < 1 %
# of each draw, and fp32 accumulation and the exponential (2^-22) add 1e-6 to 2e-3.
SLACK = 1.04
NAMES = ("out", "dq", "dk", "dv")


def _host_case(lens, hq, hk, d):
    import torch
    g = torch.Generator().manual_seed(sum(lens) + hq)
    n = sum(lens)
    t = [torch.randn(n, h, d, generator=g).to(torch.bfloat16) for h in (hq, hk, hk, hq)]
    return t, [0] + [int(c) for c in np.cumsum(lens)]


def _errors(got, want):
    return [np.linalg.norm(a - b) / np.linalg.norm(b) for a, b in zip(got, want)]


def _exact(t, cu, scale, causal):
    q, k, v, do = t
    return (blocks.attention_forward(q, k, v, cu, scale, causal)[0], *blocks.attention_backward(q, k, v, do, cu, scale, causal)[0])


@pytest.mark.parametrize("lens,hq,hk,d,scale,causal", CASES)
def test_limits_tell_planted_mistakes(lens, hq, hk, d, scale, causal):
    t, cu = _host_case(lens, hq, hk, d)
    t = [x.double().numpy() for x in t]
    want = _exact(t, cu, scale, causal)
    base = _errors(blocks.attention_rounded(*t, cu, scale, causal), want)
    assert all(1e-3 < e < 3e-3 for e in base)
    for mistake, i in (("dropped", 2), ("negated", 2), ("one number", 1)):
        e = _errors(blocks.attention_rounded(*t, cu, scale, causal, mistake), want)
        assert e[i] > SLACK * base[i], (mistake, e[i], base[i])


@pytest.mark.gpu
@pytest.mark.parametrize("lens,hq,hk,d,scale,causal", CASES)
def test_errors_are_those_of_the_documented_roundings(lens, hq, hk, d, scale, causal):
    from gpu_util import to_host
    from test_attention_gpu import _object
    t, cu = _host_case(lens, hq, hk, d)
    q, k, v, do = (x.cuda() for x in t)
    a = _object(cu, hq, hk, d, "bf16", causal, scale=scale)
    out, lse = a.forward(q, k, v)
    got = [to_host(x) for x in (out, *a.backward(do, q, k, v, out, lse))]
    a.poll()
    t = [x.double().numpy() for x in t]
    want = _exact(t, cu, scale, causal)
    limits = _errors(blocks.attention_rounded(*t, cu, scale, causal), want)
    for name, e, limit in zip(NAMES, _errors(got, want), limits):
        assert e <= SLACK * limit, (name, e, limit)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,hq,hk,d,scale,causal", CASES)
def test_errors_in_fp32(lens, hq, hk, d, scale, causal):
    # the package's fp32 criterion: relative Frobenius error 1e-5
    from gpu_util import to_host
    from test_attention_gpu import _object
    t, cu = _host_case(lens, hq, hk, d)
    q, k, v, do = (x.float().cuda() for x in t)
    a = _object(cu, hq, hk, d, "fp32", causal, scale=scale)
    out, lse = a.forward(q, k, v)
    got = [to_host(x) for x in (out, *a.backward(do, q, k, v, out, lse))]
    t = [x.double().numpy() for x in t]
    for name, e in zip(NAMES, _errors(got, _exact(t, cu, scale, causal))):
        assert e <= 1e-5, (name, e)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,hq,hk,d,causal,path", [
    ((6,), 64, 8, 128, True, 0), ((6,) * 30, 8, 1, 64, True, 0), ((3,) * 50, 12, 4, 64, False, 0), ((1, 2) * 40, 16, 16, 64, True, 0),
    ((40,), 32, 8, 128, True, 0), ((128, 17, 100), 10, 2, 96, False, 0), ((64, 128, 1, 33), 4, 4, 40, True, 0),
    ((6,) * 30, 8, 1, 64, True, 1), ((3,) * 50, 12, 4, 64, False, 1), ((40, 64, 17), 8, 2, 128, True, 1), ((64, 1, 33), 3, 3, 40, False, 1),
])
def test_query_gradient_of_short_sequences_is_off_by_its_own_rounding(lens, hq, hk, d, causal, path):
    # sequences of at most one block of keys (128, on plain FMA 64): delta is summed from P and dP in fp32, dS enters as
    # two bf16 numbers (2^-16), so that dq is the exact gradient, rounded once.  Its error is that rounding's, up to the
    # share that fp32 sums and the exponential add (under 2^-16 of the terms of dS, which cancel to a tenth in the worst
    # row: 2e-4 in all)
    from gpu_util import to_host
    from test_attention_gpu import _object
    t, cu = _host_case(lens, hq, hk, d)
    q, k, v, do = (x.cuda() for x in t)
    a = _object(cu, hq, hk, d, "bf16", causal, path=path)
    out, lse = a.forward(q, k, v)
    dq = to_host(a.backward(do, q, k, v, out, lse)[0])
    a.poll()
    t = [x.double().numpy() for x in t]
    want = blocks.attention_backward(*t, cu, d ** -0.5, causal)[0][0]
    rounding = _errors([blocks._bf16(want)], [want])[0]
    assert _errors([dq], [want])[0] <= rounding + 2e-4
