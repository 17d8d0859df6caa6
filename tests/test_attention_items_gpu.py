"""Packed attention in bf16 on the GPU with several work items per SM: the second and later turns of every barrier, of the
work feed and of the tail warp, against 64 bits in every element."""
import numpy as np
import pytest

from test_attention_gpu import _check, _object, _tensors

pytestmark = pytest.mark.gpu


def _items(lens, hq, hk):
    """Work items of the forward, the query gradient and the key / value gradient (128-row tiles)."""
    t = 128 // (hq // hk)
    return [hk * sum(-(-n // s) for n in lens) for s in (2 * t, t, 128)]


RAGGED = tuple(int(n) for n in np.random.default_rng(3).integers(1, 420, 48))
# four lengths in turn: a full tile, a short one, a tail inside the 16-row step, one on it
MIXED = (128, 5, 261, 144) * 40


@pytest.mark.parametrize("lens,hq,hk,d,causal,items", [
    ((616,) * 8, 32, 8, 128, True, 320),           # the tuning batch
    ((577,) * 8, 16, 16, 64, False, 380),          # the vision tower
    (RAGGED, 10, 2, 96, True, 180),                # dirty tails of every length, groups of 5
    (RAGGED, 28, 4, 128, False, 360),
    (MIXED, 4, 4, 64, True, 700),
    (MIXED, 6, 2, 40, False, 300),
    ((7, 16) * 300, 2, 2, 128, True, 1000),        # items of one block: every barrier turns once per item
])
def test_several_items_per_sm_against_64_bits(lens, hq, hk, d, causal, items):
    assert min(_items(lens, hq, hk)) >= items > 148
    q, k, v, do, cu = _tensors(len(lens) + hq, lens, hq, hk, d, "bf16")
    _check(_object(cu, hq, hk, d, "bf16", causal), q, k, v, do, cu, d ** -0.5, causal, "bf16")


def test_calls_of_one_object_at_once_on_two_streams():
    # both streams always have work, of this object and of the layer norm; each call has its own scratch
    import torch
    import paper_2503_21817_b200 as sk
    lens, hq, hk, d = (300, 41, 577, 128, 5), 8, 2, 64
    q, k, v, do, cu = _tensors(41, lens, hq, hk, d, "bf16")
    a = _object(cu, hq, hk, d, "bf16")
    gamma = torch.ones(hq * d, dtype=torch.bfloat16, device="cuda")

    def step():
        out, lse = a.forward(q, k, v)
        y, mean, rstd = sk.layernorm_forward(out.view(len(out), -1), gamma)
        dx, dgamma, dbeta = sk.layernorm_backward(do.view(len(out), -1), out.view(len(out), -1), gamma, mean, rstd)
        return (out, lse, y, dx, dgamma, dbeta, *a.backward(dx.view_as(out), q, k, v, out, lse))

    want = step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(25):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(step())
    torch.cuda.synchronize()
    a.poll()
    assert all(torch.equal(x, y) for g in got for x, y in zip(g, want))
