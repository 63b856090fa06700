"""Attention over 4-bit caches where a CTA has many short pieces, and where blocks' ids are bad: the answer is the one over a block of zeros in
the bad one's place, bit for bit and every time (both calls do the same arithmetic in the same order)."""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_cache import rand
from test_gpu_cache4 import Setup

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


@pytest.mark.parametrize("heads,group,dim,bs,new,layout", [(8, 4, 128, 16, 1, 0), (2, 4, 128, 8, 1, 1), (8, 4, 128, 5, 1, 0), (2, 8, 64, 3, 2, 1), (1, 2, 256, 16, 5, 0), (4, 2, 96, 32, 3, 0),
                                                           (2, 4, 128, 16, 20, 0)])
def test_bad_blocks_are_blocks_of_zeros_in_every_piece(heads, group, dim, bs, new, layout):
    rng = np.random.default_rng(heads + dim + bs)
    context = rng.integers(0, 260, 500 if new < 20 else 60).tolist()
    s = Setup("e2m1", heads, dim, bs, context, [new] * len(context), layers=1, layout=layout, seed=bs)
    s.fill()
    q = rand(s, s.tokens, heads * group, dim)
    spare = (set(range(s.nb)) - {int(x) for r, c in enumerate(context) for x in s.host_tables[r, :-(-(c + new) // bs)]}).pop()
    blocks = s.pool.view(1, 2, s.nb, -1) if layout == kvr.LAYER_MAJOR else s.pool.view(s.nb, 1, 2, -1).permute(1, 2, 0, 3)
    blocks[:, :, spare] = 0
    bad, zero = s.host_tables.copy(), s.host_tables.copy()
    for r in range(len(context)):
        for i in rng.integers(0, -(-(context[r] + new) // bs), 2):
            bad[r, i], zero[r, i] = rng.choice([s.nb, -1, -2**31, 2**31 - 1]), spare
    workspace = torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")

    def attend(table):
        out, lse = torch.zeros_like(q), torch.zeros(s.tokens, heads * group, device="cuda")
        s.status.zero_()
        batch = kvr.Batch(s.arrays[0], s.arrays[1], torch.from_numpy(table).cuda(), new, max(context) + new, s.status)
        s.cache.attend(s.pool, 0, batch, q, out, workspace, lse=lse)
        torch.cuda.synchronize()
        return out, lse, int(s.status)

    want, want_lse, status = attend(zero)
    assert status == 0 and torch.isfinite(want).all()
    for _ in range(5):
        out, lse, status = attend(bad)
        assert status == kvr.DEV_BAD_BLOCK and torch.equal(out, want) and torch.equal(lse, want_lse)
