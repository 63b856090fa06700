"""Block tables that are columns of wider ones."""
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_cache import Setup, rand

pytestmark = pytest.mark.gpu


def test_a_request_longer_than_its_part_of_a_table_is_left_out():
    """The columns behind a cut table hold other things; here they are valid blocks, which only the length keeps from being used."""
    s = Setup("bf16", 2, 64, 16, [40, 20, 100], [2, 2, 2], layers=1, seed=3)
    s.fill()
    q, ws = rand(s, 6, 4, 64), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    want = torch.zeros_like(q)
    s.cache.attend(s.pool, 0, s.batch, q, want, ws)
    s.ok()
    cut = kvr.Batch(s.arrays[0], s.arrays[1], s.arrays[2][:, :3], 2, 102, s.status)      # 48 tokens; the last request has 102
    out = torch.full_like(q, 3.0)
    s.cache.attend(s.pool, 0, cut, q, out, ws)
    torch.cuda.synchronize()
    assert int(s.status) == kvr.DEV_BAD_LENGTH and torch.equal(out[:4], want[:4]) and (out[4:] == 3).all()
    before = s.pool.clone()
    for call in (lambda: s.cache.append(s.pool, 0, cut, k=rand(s, 6, 2, 64)),
                 lambda: s.cache.keep(s.pool, cut, torch.tensor([[1]] * 3, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda"))):
        s.status.zero_()
        s.pool.copy_(before)
        call()
        torch.cuda.synchronize()
        assert int(s.status) == kvr.DEV_BAD_LENGTH
        rows, old = s.plane(0, 0), s.plane(0, 0, before)
        assert torch.equal(rows[s.slots(2, 0, 102)], old[s.slots(2, 0, 102)]) and not torch.equal(rows, old)
    k = torch.full((6, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    s.status.zero_()
    s.cache.read(s.pool, 0, cut, k=k)
    torch.cuda.synchronize()
    assert int(s.status) == kvr.DEV_BAD_LENGTH and (k[4:] == 3).all() and not (k[:4] == 3).all(-1).any()


def test_a_part_of_a_step_is_attended_to_and_kept_by_itself():
    """Requests 1 and 2 of three as a batch of their own, their rows where they are among the step's."""
    s = Setup("bf16", 2, 64, 16, [40, 20, 100], [5, 4, 6], layers=2, seed=4)
    s.fill(0)
    s.fill(1)
    q, ws = rand(s, 15, 4, 64), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    want, out = torch.zeros_like(q), torch.full_like(q, 3.0)
    s.cache.attend(s.pool, 0, s.batch, q, want, ws)
    part = kvr.Batch(s.arrays[0][1:], s.arrays[1][1:], s.arrays[2][1:], 6, 106, s.status)
    s.cache.attend(s.pool, 0, part, q, out, ws)
    s.ok()
    assert torch.equal(out[5:], want[5:]) and (out[:5] == 3).all()
    index = torch.tensor([[1, 4], [1, 3], [0, 5]], dtype=torch.int32, device="cuda")
    count = torch.tensor([0, 2, 2], dtype=torch.int32, device="cuda")
    before = s.pool.clone()
    s.cache.keep(s.pool, s.batch, index, count)
    s.ok()
    want = s.pool.clone()
    s.pool.copy_(before)
    s.cache.keep(s.pool, part, index[1:], count[1:])
    s.ok()
    assert torch.equal(s.pool, want) and not torch.equal(want, before)
