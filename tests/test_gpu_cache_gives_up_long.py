"""Attention whose waits run out while loads are under way, over contexts that keep every buffer busy: the call ends with the status, writes nothing
but its outputs and workspace, and the next one is right."""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_cache import KIND, rand, tree
from test_gpu_cache4 import Setup

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


@pytest.mark.parametrize("fmt,heads,group,dim,bs,new", [("e2m1", 8, 4, 128, 16, 1), ("e2m1", 8, 4, 128, 5, 1), ("e2m1", 2, 2, 256, 8, 4), ("e2m1", 2, 4, 128, 16, 20), ("e2m1", 2, 8, 128, 8, 40),
                                                        ("bf16", 2, 4, 128, 16, 20), ("bf16", 2, 8, 64, 8, 40), ("f16", 2, 8, 128, 16, 40), ("e4m3", 2, 8, 128, 16, 20), ("int8", 2, 8, 64, 8, 40)])
def test_waits_that_run_out_under_load(fmt, heads, group, dim, bs, new):
    s = Setup(fmt, heads, dim, bs, [6000, 11000, 300, 7000], [new] * 4, layers=1, seed=new + dim)
    s.fill()
    mask, _ = tree(s, np.random.default_rng(new))
    q = rand(s, s.tokens, heads * group, dim, dtype=KIND["f16" if fmt == "f16" else "bf16"])
    pool = s.pool.clone()

    def attend():
        out, ws = torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        s.status.zero_()
        s.cache.attend(s.pool, 0, s.batch, q, out, ws, mask=mask)
        torch.cuda.synchronize()
        return out, int(s.status)

    want, status = attend()
    assert status == 0
    polls = kvr.lib().kvr_test_attend_polls
    for limit in (1, 2, 3, 5, 9, 17, 33, 65, 129):
        was = polls(limit)
        try:
            out, status = attend()
        finally:
            polls(was)
        assert status in (0, kvr.DEV_GAVE_UP) and (status or torch.equal(out, want))
    out, status = attend()
    assert status == 0 and torch.equal(out, want) and torch.equal(s.pool, pool)
