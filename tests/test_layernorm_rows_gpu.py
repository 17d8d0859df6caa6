"""Layer norm backward on the GPU with several rows per row group: the ring of copies, the alternating sums and the
gradients summed over a group's rows, against 64 bits in every element."""
import pytest

from test_layernorm_gpu import _case, _within, blocks, to_host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,C", [
    (9001, 40),            # 20 groups per CTA: 2960 groups
    (6007, 1024),          # 10: 1480
    (4003, 1664),          # 5 (a part-filled warp): 740
    (1501, 5120),          # 2: 296
    (701, 6144),           # 1: 148
    (603, 10240),          # 1, the widest row held in registers
    (403, 10248),          # the two-kernel form
])
def test_several_rows_per_group_against_64_bits(n, C, dtype):
    import torch
    import paper_2503_21817_b200 as sk
    x, gamma, beta, dy = _case(n + C, n, C, dtype, 0.5)
    y, mean, rstd = sk.layernorm_forward(x, gamma, beta)
    X, g, b, G = (to_host(t) for t in (x, gamma, beta, dy))
    r = blocks.layernorm_forward(X, g, b, 1e-5, dtype)
    for name, got, want, err in zip(("y", "mean", "rstd"), (y, mean, rstd), r[:3], r[3:]):
        _within(got, want, err, name)
    M, R = to_host(mean), to_host(rstd)
    grads = sk.layernorm_backward(dy, x, gamma, mean, rstd, dw_fp32=True)
    refs, errs = blocks.layernorm_backward(G, X, g, M, R, dtype, "fp32")
    for name, got, want, err in zip(("dx", "dgamma", "dbeta"), grads, refs, errs):
        _within(got, want, err, name)
    again = sk.layernorm_backward(dy, x, gamma, mean, rstd, dw_fp32=True)
    assert all(torch.equal(p, q) for p, q in zip(grads, again))
