"""Layer normalisation on the GPU against its fp64 statement, and the blocks it is used in."""
import numpy as np
import pytest

from oracle import blocks
from gpu_util import to_host

pytestmark = pytest.mark.gpu


def _case(seed, n, C, dtype, offset=0.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (torch.randn(n, C, generator=g) * (0.2 + torch.rand(n, 1, generator=g)) + offset).to(dt).cuda()
    return x, *((torch.randn(*s, generator=g) * f + o).to(dt).cuda() for s, f, o in (((C,), 0.2, 1.0), ((C,), 0.2, 0.0), ((n, C), 1.0, 0.0)))


def _within(got, want, bound, what):
    got = to_host(got)
    assert np.isfinite(got).all(), what
    worst = np.max(np.abs(got - want) / np.maximum(bound, 1e-300)) if got.size else 0.0
    assert worst <= 1.0, f"{what}: an element is {worst:.3f} times its bound away"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,C,offset", [
    (1, 8, 0.0), (3, 264, 0.0), (577, 1024, 0.0), (1000, 40, 5.0), (301, 1664, 0.0),
    (40, 5120, 0.0), (40, 6144, 3.0), (9, 8192, 0.0), (5, 12296, 0.0), (3, 16384, 0.0),
    (64, 1024, 300.0),                     # deviations far below the mean
])
def test_against_64_bits(n, C, offset, dtype):
    import torch
    import paper_2503_21817_b200 as sk
    x, gamma, beta, dy = _case(n + C, n, C, dtype, offset)
    y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
    X, g, b, G = (to_host(t) for t in (x, gamma, beta, dy))
    r = blocks.layernorm_forward(X, g, b, 1e-5, dtype)
    for name, got, want, err in zip(("y", "mean", "rstd"), (y, mean, rstd), r[:3], r[3:]):
        _within(got, want, err, name)
    M, R = to_host(mean), to_host(rstd)
    for fp32 in (False, True):
        grads = sk.layernorm_backward(dy, x, gamma, mean, rstd, dw_fp32=fp32)
        refs, errs = blocks.layernorm_backward(G, X, g, M, R, dtype, "fp32" if fp32 else None)
        for name, got, want, err in zip(("dx", "dgamma", "dbeta"), grads, refs, errs):
            _within(got, want, err, name)
        again = sk.layernorm_backward(dy, x, gamma, mean, rstd, dw_fp32=fp32)
        assert all(torch.equal(p, q) for p, q in zip(grads, again))
    # in place, without beta
    y0, *_ = sk.layernorm_forward(x, gamma)
    z = x.clone()
    assert torch.equal(sk.layernorm_forward(z, gamma, out=z)[0], y0) and torch.equal(z, y0)
    d = dy.clone()
    sk.layernorm_backward(d, x, gamma, mean, rstd, dx=d)
    assert torch.equal(d, grads[0])
    d = x.clone()
    g2 = sk.layernorm_backward(dy, d, gamma, mean, rstd, dx=d, dw_fp32=True)
    assert torch.equal(d, grads[0]) and torch.equal(g2[1], grads[1])


def test_gradient_against_differences():
    # central differences of the 64-bit forward are exact to about 1e-8 here; the fp32 kernels' sums err by
    # less than 2e-5 of their absolute terms (oracle/blocks.py)
    import paper_2503_21817_b200 as sk
    x, gamma, beta, dy = _case(1, 33, 264, "fp32", 1.0)
    y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
    grads = [to_host(t) for t in sk.layernorm_backward(dy, x, gamma, mean, rstd)]
    host, G, r = [to_host(t) for t in (x, gamma, beta)], to_host(dy), np.random.default_rng(0)
    f = lambda *t: float(np.sum(G * blocks.layernorm_forward(*t, 1e-5, "fp32")[0]))
    for i in range(3):
        e = r.standard_normal(host[i].shape)
        moved = lambda s: [t + s * e if j == i else t for j, t in enumerate(host)]
        num = (f(*moved(1e-4)) - f(*moved(-1e-4))) / 2e-4
        assert abs(num - np.sum(grads[i] * e)) <= 2e-5 * np.abs(grads[i] * e).sum() + 1e-5


def test_rows_stay_apart_and_no_rows():
    import torch
    import paper_2503_21817_b200 as sk
    x, gamma, beta, dy = _case(2, 50, 512, "bf16")
    y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
    bad = x.clone()
    bad[7] = float("nan")
    y2, mean2, rstd2 = sk.layernorm_forward(bad, gamma, beta)
    keep = torch.arange(50, device="cuda") != 7
    assert torch.equal(y[keep], y2[keep]) and bool(torch.isnan(y2[7]).all())
    dx, dx2 = (sk.layernorm_backward(dy, t, gamma, m, r)[0] for t, m, r in ((x, mean, rstd), (bad, mean2, rstd2)))
    assert torch.equal(dx[keep], dx2[keep])
    e, m, r = sk.layernorm_forward(x[:0], gamma, beta)
    assert e.shape == (0, 512) and m.shape == (0,)
    dx, dg, db = sk.layernorm_backward(dy[:0], x[:0], gamma, m, r)
    assert dx.shape == (0, 512) and not dg.any() and not db.any()
    # a row of equal values: zero deviations, rstd = eps^-1/2
    flat = torch.full((2, 64), 3.0, dtype=torch.float32, device="cuda")
    w = torch.ones(64, device="cuda")
    y, _, rstd = sk.layernorm_forward(flat, w, w * 0.5)
    assert bool((y == 0.5).all()) and np.allclose(to_host(rstd), 1e-5 ** -0.5, rtol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("power", [-60, 58])
def test_gradient_scales_with_tiny_and_huge_rows(dtype, power):
    # eps = 0: x -> 2^p x keeps y and dgamma, divides dx by 2^p, exactly but for products that leave the normal
    # numbers of fp32: xh, rstd m and rstd t stay in them here, rstd^2 would not
    import torch
    import paper_2503_21817_b200 as sk
    x, gamma, beta, dy = _case(5, 20, 1024, dtype)
    a, b = ((s, *sk.layernorm_forward(s, gamma, beta, eps=0.0)) for s in (x, x * 2.0 ** power))
    assert torch.equal(a[1], b[1])
    ga, gb = (sk.layernorm_backward(dy, t[0], gamma, t[2], t[3]) for t in (a, b))
    assert torch.equal(ga[0], gb[0] * 2.0 ** power) and torch.equal(ga[1], gb[1]) and torch.equal(ga[2], gb[2])


def test_elements_past_32_bits():
    # 2^31 elements and some rows: the last rows are those of a call with only them; the others' gradient is zero
    import torch
    import paper_2503_21817_b200 as sk
    n, C, k = (1 << 31) // 4096 + 5, 4096, 9
    x, gamma, beta, dy = _case(4, k, C, "bf16")
    big, d = (torch.zeros(n, C, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    big[-k:], d[-k:] = x, dy
    y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
    Y, M, R = sk.layernorm_forward(big, gamma, beta)
    assert torch.equal(Y[-k:], y) and torch.equal(M[-k:], mean) and torch.equal(R[-k:], rstd) and torch.equal(Y[0], beta)
    del Y
    dx, dg, db = sk.layernorm_backward(d, big, gamma, M, R, dw_fp32=True, dx=d)
    want = sk.layernorm_backward(dy, x, gamma, mean, rstd)[0]
    assert torch.equal(dx[-k:], want) and not dx[:-k].any()
    refs, errs = blocks.layernorm_backward(*(to_host(t) for t in (dy, x, gamma, mean, rstd)), "bf16", "fp32")
    for name, got, r, e in zip(("dgamma", "dbeta"), (dg, db), refs[1:], errs[1:]):       # sums of zeros add no error
        _within(got, r, e, name)


def test_refusals():
    import torch
    import paper_2503_21817_b200 as sk
    x, gamma, beta, dy = _case(3, 6, 64, "bf16")
    for a in ((x.half(), gamma, beta), (x.t(), gamma, beta), (x, gamma.float(), beta), (x, gamma[:32], beta), (x, gamma, beta.cpu()),
              (x.cpu(), gamma, beta)):
        with pytest.raises(ValueError):
            sk.layernorm_forward(*a)
    with pytest.raises(sk.SkipFFNError):
        sk.layernorm_forward(x[:, :12].contiguous(), gamma[:12].contiguous(), None)
    buf = torch.zeros(7, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sk.SkipFFNError):
        sk.layernorm_forward(buf[:6], gamma, beta, out=buf[1:])           # half over the input
    y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
    for a in ((dy[:3], x, gamma, mean, rstd), (dy, x, gamma, mean[:3], rstd), (dy, x, gamma, mean.double(), rstd), (dy.float(), x, gamma, mean, rstd)):
        with pytest.raises(ValueError):
            sk.layernorm_backward(*a)


@pytest.mark.parametrize("capture", [False, True])
def test_block_of_norm_attention_and_skip_ffn(capture):
    """The blocks as they are used: x + proj(attention(qkv(norm x))) and then the Skip-FFN sublayer, forward and
    backward, in fp32 against autograd in 64 bits; captured into a graph and replayed it gives the same bits.
    The criterion is the package's fp32 one (relative Frobenius error 1e-5) for each result."""
    import torch
    import paper_2503_21817_b200 as sk
    lens, C, I, hq, hk, d = (90, 1, 150), 128, 256, 4, 2, 32
    n, cu = sum(lens), [0, 90, 91, 241]
    g = torch.Generator().manual_seed(0)
    rand = lambda *s, f=1.0: (torch.randn(*s, generator=g) * f).cuda()
    x, dout = rand(n, C), rand(n, C)
    gamma, beta, Wqkv, Wo = 1 + rand(C, f=0.1), rand(C, f=0.1), rand((hq + 2 * hk) * d, C, f=0.09), rand(C, hq * d, f=0.09)
    Wg, Wu, Wd = rand(I, C, f=0.09), rand(I, C, f=0.09), rand(C, I, f=0.06)
    mask = (torch.rand(n, generator=g) < 0.6).to(torch.uint8).cuda()
    attn = sk.PackedAttention(cu, hq, hk, d, dtype=sk.FP32)
    ffn = sk.SkipFFN(C, I, n, dtype=sk.FP32)

    def step():
        y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
        qkv = (y @ Wqkv.t()).view(n, hq + 2 * hk, d)
        q, k, v = qkv.split((hq, hk, hk), 1)
        o, lse = attn.forward(q, k, v)
        h = x + o.view(n, -1) @ Wo.t()
        out = ffn.forward(h, mask, Wg, Wu, Wd)
        dh, dWg, dWu, dWd = ffn.backward(dout)
        do = (dh @ Wo).view(n, hq, d)
        dqkv = torch.empty_like(qkv)
        attn.backward(do, q, k, v, o, lse, *dqkv.split((hq, hk, hk), 1))
        dqkv2 = dqkv.view(n, -1)
        dx, dgamma, dbeta = sk.layernorm_backward(dqkv2 @ Wqkv, x, gamma, mean, rstd)
        return out, dx + dh, dgamma, dbeta, dqkv2.t() @ y, dh.t() @ o.view(n, -1), dWg, dWu, dWd

    got = step()
    ffn.poll()
    attn.poll()
    if capture:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, cap))
        return
    X, ga, be, W1, W2, G1, U1, D1 = leaves = [t.double().requires_grad_() for t in (x, gamma, beta, Wqkv, Wo, Wg, Wu, Wd)]
    y = (X - X.mean(1, keepdim=True)) / torch.sqrt(X.var(1, unbiased=False, keepdim=True) + 1e-5) * ga + be
    q, k, v = (y @ W1.t()).view(n, hq + 2 * hk, d).split((hq, hk, hk), 1)
    rows = []
    for a, b in zip(cu, cu[1:]):
        late = torch.ones(b - a, b - a, device="cuda").triu(1).bool()
        s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b].repeat_interleave(hq // hk, 1)) * d ** -0.5
        rows.append(torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(late, -float("inf")), -1), v[a:b].repeat_interleave(hq // hk, 1)))
    h = X + torch.cat(rows).reshape(n, -1) @ W2.t()
    f = (torch.nn.functional.silu(h @ G1.t()) * (h @ U1.t())) @ D1.t()
    out = torch.where(mask[:, None] != 0, h, h + f)
    want = (out, *torch.autograd.grad(out, leaves, dout.double()))
    for i, (a, b) in enumerate(zip(got, want)):
        err = ((a.double() - b).norm() / b.norm()).item()
        assert err <= 1e-5, (i, err)
