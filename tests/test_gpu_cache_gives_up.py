"""The tile kernel's bounded waits: when one runs out the call ends with KVR_DEV_GAVE_UP and the next one is right.

The limit is lowered on the host; the waits are the kernel's ordinary ones, on barriers that do complete later.
"""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_cache import KIND, Setup, rand, tree

pytestmark = pytest.mark.gpu


@pytest.fixture
def polls():
    """Sets the limit; the library's own is back afterwards."""
    was = kvr.lib().kvr_test_attend_polls(1 << 18)
    kvr.lib().kvr_test_attend_polls(was)
    yield kvr.lib().kvr_test_attend_polls
    torch.cuda.synchronize()
    kvr.lib().kvr_test_attend_polls(was)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("heads,group,dim,bs,new", [(2, 4, 128, 16, 20), (2, 8, 128, 8, 40), (2, 8, 64, 5, 10)])
def test_a_call_that_gives_up_says_so_and_the_next_is_right(polls, fmt, dtype, heads, group, dim, bs, new):
    s = Setup(fmt, heads, dim, bs, [900, 30, 0], [new] * 3, layers=1, seed=new)
    s.fill()
    mask, _ = tree(s, np.random.default_rng(new))
    q = rand(s, s.tokens, heads * group, dim, dtype=KIND[dtype])

    def attend():
        out, ws = torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        s.status.zero_()
        s.cache.attend(s.pool, 0, s.batch, q, out, ws, mask=mask)
        torch.cuda.synchronize()
        return out, int(s.status)

    want, status = attend()
    assert status == 0
    for limit in (0, 1, 8, 100):
        was = polls(limit)
        out, status = attend()
        assert status == kvr.DEV_GAVE_UP if limit == 0 else status in (0, kvr.DEV_GAVE_UP)
        assert status or torch.equal(out, want)
        polls(was)
        out, status = attend()
        assert status == 0 and torch.equal(out, want)
