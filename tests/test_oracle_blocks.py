"""The fp64 statements of packed attention and layer normalisation, pinned on the CPU: special cases with known
answers, gradients against central differences."""
import numpy as np
import pytest

from oracle import blocks


def _inputs(seed, lens, hq, hk, d):
    r = np.random.default_rng(seed)
    n = sum(lens)
    cu = np.concatenate([[0], np.cumsum(lens)])
    return r.standard_normal((n, hq, d)), r.standard_normal((n, hk, d)), r.standard_normal((n, hk, d)), r.standard_normal((n, hq, d)), cu


def test_single_token_and_first_row():
    q, k, v, do, cu = _inputs(0, (1, 4), 4, 2, 8)
    out, lse, *_ = blocks.attention_forward(q, k, v, cu, 0.3, True)
    for h in range(4):
        for t in (0, 1):                                       # first token of either sequence sees itself only
            assert np.allclose(out[t, h], v[t, h // 2])
            assert np.isclose(lse[t, h], 0.3 * q[t, h] @ k[t, h // 2])
    (dq, dk, dv), _ = blocks.attention_backward(q, k, v, do, cu, 0.3, True)
    assert np.allclose(dq[0], 0) and np.allclose(dk[0], 0)
    assert np.allclose(dv[0, 0], do[0, 0] + do[0, 1])


def test_equal_scores_average_and_causal_is_a_prefix():
    q, k, v, _, cu = _inputs(1, (6,), 1, 1, 8)
    out, lse, *_ = blocks.attention_forward(0 * q, k, v, cu, 1.0, False)
    assert np.allclose(out[:, 0], v[:, 0].mean(0)) and np.allclose(lse, np.log(6))
    whole = blocks.attention_forward(q, k, v, cu, 0.5, True)[0]
    for t in range(6):
        part = blocks.attention_forward(q[:t + 1], k[:t + 1], v[:t + 1], [0, t + 1], 0.5, False)[0]
        assert np.allclose(whole[t], part[t])


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradient_against_differences(causal):
    q, k, v, do, cu = _inputs(2, (5, 1, 3), 4, 2, 8)
    args = [q, k, v]
    grads, _ = blocks.attention_backward(q, k, v, do, cu, 0.4, causal)
    r = np.random.default_rng(3)
    for i in range(3):
        for _ in range(3):
            e = r.standard_normal(args[i].shape)
            f = lambda s: np.sum(do * blocks.attention_forward(*[a + s * e if j == i else a for j, a in enumerate(args)], cu, 0.4, causal)[0])
            # central differences in 64 bits: h^2 f''' / 6 plus 2^-52 |f| / h, both far below 1e-7 |f'| scale
            num = (f(1e-4) - f(-1e-4)) / 2e-4
            assert abs(num - np.sum(grads[i] * e)) <= 1e-5 * (1 + np.abs(grads[i] * e).sum())


def test_layernorm_against_its_definition_and_differences():
    r = np.random.default_rng(4)
    x, g, b, dy = r.standard_normal((5, 16)) * 3 + 1, r.standard_normal(16), r.standard_normal(16), r.standard_normal((5, 16))
    y, mean, rstd, *_ = blocks.layernorm_forward(x, g, b, 1e-5)
    z = (y - b) / g
    assert np.allclose(z.mean(1), 0) and np.allclose((z * z).mean(1), 1, atol=1e-4)
    (dx, dg, db), _ = blocks.layernorm_backward(dy, x, g, mean, rstd)
    f = lambda x, g, b: np.sum(dy * blocks.layernorm_forward(x, g, b, 1e-5)[0])
    for i, grad in enumerate((dx, dg, db)):
        a = [x, g, b]
        e = r.standard_normal(a[i].shape)
        up, down = list(a), list(a)
        up[i], down[i] = a[i] + 1e-4 * e, a[i] - 1e-4 * e
        assert abs((f(*up) - f(*down)) / 2e-4 - np.sum(grad * e)) <= 1e-5 * (1 + np.abs(grad * e).sum())
