"""The bounded waits of the tensor-core attention kernels: one that runs out ends the call with a status, and the
context, the object and its work lists stay usable."""
import time

import pytest

from test_attention_gpu import _object, _tensors

pytestmark = pytest.mark.gpu

ETIMEOUT = 5
SITES = range(1, 8)


@pytest.mark.parametrize("lens,hq,hk,d,causal", [
    ((300, 129), 8, 2, 128, True),
    ((300, 129), 2, 2, 64, False),
    ((616,) * 8, 32, 8, 128, True),            # every SM has a CTA that gives up, with further items to come
])
def test_expired_wait_is_reported_and_the_context_stays_usable(lens, hq, hk, d, causal):
    import torch
    import paper_2503_21817_b200 as sk
    q, k, v, do, cu = _tensors(31, lens, hq, hk, d, "bf16")
    a = _object(cu, hq, hk, d, "bf16", causal)
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    a.poll()
    calls = (lambda: a.forward(q, k, v), lambda: a.backward(do, q, k, v, out, lse))
    for call in calls:
        a.tune(wait_us=2000, lose_load=1)      # key tiles announce bytes that never come
        t0 = time.perf_counter()
        call()
        with pytest.raises(sk.SkipFFNError) as e:
            a.poll()
        assert time.perf_counter() - t0 < 0.5
        assert e.value.status == ETIMEOUT and any(f"site {s})" in str(e.value) for s in SITES)
        a.poll()                               # reported once
        a.tune(wait_us=1000000, lose_load=0)
        out2, lse2 = a.forward(q, k, v)
        grads2 = a.backward(do, q, k, v, out2, lse2)
        a.poll()
        assert all(torch.equal(x, y) for x, y in zip((out, lse, *grads), (out2, lse2, *grads2)))


def test_knobs_outside_their_ranges_are_refused():
    import paper_2503_21817_b200 as sk
    a = _object([0, 8], 2, 2, 64, "bf16")
    for knob in (dict(wait_us=0), dict(wait_us=-1), dict(wait_us=4000001), dict(lose_load=2), dict(lose_load=-1)):
        with pytest.raises(sk.SkipFFNError):
            a.tune(**knob)
    assert [a.lib.skipffn_attention_tune(a._handle, w, 1) for w in (-1, 2)] == [1, 1]
    with pytest.raises(KeyError):
        a.tune(other=1)
    a.tune(wait_us=1)
    a.tune(wait_us=4000000, lose_load=0)


@pytest.mark.parametrize("lens,hq,hk,d", [
    # a long sequence and a short one with a part-filled 16-row step: the warp that zeroes tails has nothing to do
    # until the CTA has been through the long one
    ((32768, 7), 16, 16, 64),
    # items of one row tile, then items of two: the second tile's softmax warps have nothing to do until then
    ((32,) * 30000 + (64,) * 300, 16, 4, 8),
])
def test_a_wait_may_take_longer_than_its_limit_while_the_kernel_moves_on(lens, hq, hk, d):
    import torch
    q, k, v, do, cu = _tensors(32, lens, hq, hk, d, "bf16")
    a = _object(cu, hq, hk, d, "bf16")
    out, lse = a.forward(q, k, v)
    grads = a.backward(do, q, k, v, out, lse)
    a.poll()
    limit = 0.5
    t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.tune(wait_us=int(1000 * limit))
    t0.record()
    out2, lse2 = a.forward(q, k, v)
    t1.record()
    a.poll()
    assert t0.elapsed_time(t1) > 2 * limit       # milliseconds: the limit did pass in the meantime
    grads2 = a.backward(do, q, k, v, out2, lse2)
    a.poll()
    assert all(torch.equal(x, y) for x, y in zip((out, lse, *grads), (out2, lse2, *grads2)))
