"""Polling a paged cache: of its stream alone."""
import pytest

from cache_util import Batch

pytestmark = pytest.mark.gpu


def test_poll_waits_for_its_stream_alone_and_clears_before_it_returns():
    import torch
    import paper_2503_21817_b200 as sk
    x = Batch(51, (1, 1), (20, 30), 4, 2, 64, 16)
    side, busy = torch.cuda.Stream(), torch.cuda.Event()
    good = x.d_lens.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                                # the stream's memory is there before
        for _ in range(2):
            x.cache.attention(x.q)
            x.cache.poll()
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)                             # half a second or more of other work on the default stream
    busy.record()
    with torch.cuda.stream(side):
        x.d_lens[0] = -1
        x.cache.attention(x.q)
        with pytest.raises(sk.SkipFFNError, match="site 65"):
            x.cache.poll()
        x.cache.poll()                                           # reported once
        x.d_lens.copy_(good)
        x.cache.attention(x.q)
        x.cache.poll()
    assert not busy.query()
    torch.cuda.synchronize()
