"""The fp64 statements of the paged cache's operators against closed forms, differences and each other."""
import numpy as np
import pytest

from oracle import blocks, cache


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_quarter_turn_and_the_relative_position(interleaved):
    x = np.arange(8.0).reshape(1, 1, 8)
    y, _ = cache.rotary_forward(x, [[1]], [np.pi / 2] * 4, [0] * 4, 8, interleaved)
    a, b = cache.pairs_of(8, 8, interleaved)
    assert np.allclose(y[..., a], -x[..., b]) and np.allclose(y[..., b], x[..., a])
    # products of rotated vectors depend on the difference of their positions alone
    r = np.random.default_rng(0)
    q, k = r.standard_normal((2, 1, 1, 8))
    f = [1.0, 0.3, 0.1, 0.01]
    dot = lambda m, n: float(np.sum(cache.rotary_forward(q, [[m]], f, [0] * 4, 8, interleaved)[0] * cache.rotary_forward(k, [[n]], f, [0] * 4, 8, interleaved)[0]))
    assert abs(dot(7, 3) - dot(104, 100)) < 1e-12


def test_axes_rest_of_the_columns_and_norm():
    x = np.random.default_rng(1).standard_normal((3, 2, 16))
    y, _ = cache.rotary_forward(x, [[0, 5, 9], [3, 0, 0]], [1.0, 1.0], [0, 1], 4)
    assert np.array_equal(y[..., 4:], x[..., 4:])
    c = np.cos([0.0, 5.0, 9.0])[:, None]
    assert np.allclose(y[:, :, 0], x[:, :, 0] * c - x[:, :, 2] * np.sin([0.0, 5.0, 9.0])[:, None])
    assert np.allclose(y[1:, :, 1], x[1:, :, 1])               # second axis: position 0 for tokens 1 and 2
    n, _ = cache.rotary_forward(x, np.zeros((1, 3)), [], [], 0, gamma=np.full(16, 2.0), eps=0.0)
    assert np.allclose((n * n).mean(-1), 4.0)


@pytest.mark.parametrize("gamma", [True, False])
def test_rotary_gradient_against_differences(gamma):
    r = np.random.default_rng(2)
    x, dy, g = r.standard_normal((3, 2, 16)), r.standard_normal((3, 2, 16)), r.standard_normal(16) if gamma else None
    pos, f, ax = [[0, 4, 11], [7, 1, 2]], [1.0, 0.4, 0.2, 0.05], [0, 1, 0, 1]
    out = lambda x, g: float(np.sum(dy * cache.rotary_forward(x, pos, f, ax, 8, True, g)[0]))
    (dx, dg), _ = cache.rotary_backward(dy, x, pos, f, ax, 8, True, g)
    e, h = r.standard_normal(x.shape), 1e-5
    assert abs((out(x + h * e, g) - out(x - h * e, g)) / (2 * h) - np.sum(dx * e)) < 1e-8
    if gamma:
        e = r.standard_normal(16)
        assert abs((out(x, g + h * e) - out(x, g - h * e)) / (2 * h) - np.sum(dg * e)) < 1e-8


def test_attention_of_a_whole_prompt_is_causal_attention():
    r = np.random.default_rng(3)
    q, k, v = r.standard_normal((9, 4, 8)), r.standard_normal((9, 2, 8)), r.standard_normal((9, 2, 8))
    out, lse, *_ = cache.attention(q, [k], [v], [0, 9], [9], 0.3)
    o2, l2, *_ = blocks.attention_forward(q, k, v, [0, 9], 0.3, True)
    assert np.allclose(out, o2) and np.allclose(lse, l2)
    # the last two tokens alone, over the same rows; tokens that see nothing
    out, lse, *_ = cache.attention(q[7:], [k], [v], [0, 2], [9], 0.3)
    assert np.allclose(out, o2[7:])
    out, lse, *_ = cache.attention(q[:3], [k[:1]], [v[:1]], [0, 3], [1], 0.3)
    assert np.array_equal(out[:2], np.zeros((2, 4, 8))) and np.all(lse[:2] == -np.inf) and np.allclose(out[2, :2], v[0, :1])


def test_weights_of_a_token_sum_to_one_and_of_its_heads_to_their_number():
    r = np.random.default_rng(4)
    q, k = r.standard_normal((5, 6, 8)), r.standard_normal((12, 2, 8))
    _, lse, *_ = cache.attention(q, [k], [k], [0, 5], [12], 0.3)
    w, _ = cache.weights(q, [k], lse, [0, 5], [12], 2, 0.3, 15)
    assert np.allclose(w.sum(-1), 15.0) and np.all(w[..., 12:] == 0)
    w2, _ = cache.weights(q, [k], lse, [0, 5], [12], 2, 0.3, 15, prior=np.ones((1, 2, 15)))
    assert np.allclose(w2[..., :12], w[..., :12] + 1) and np.all(w2[..., 12:] == 0)


def test_evict_by_hand():
    w = np.array([0.1, 5, 3, 3, 9, 3, 0.0, np.nan, 0.2], dtype=np.float32)
    assert cache.evict(w, 9, 4, 0, 0) == [1, 2, 3, 4]            # ties to the lower row
    assert cache.evict(w, 9, 4, 1, 1) == [0, 1, 4, 8]
    assert cache.evict(w, 9, 3, 0, 3) == [6, 7, 8]
    assert cache.evict(w, 9, 8, 0, 0) == [0, 1, 2, 3, 4, 5, 6, 8]   # NaN goes first
    assert cache.evict(w, 3, 4, 0, 0) == [0, 1, 2]
