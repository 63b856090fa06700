"""Fork, resize and compact where a CUDA call of theirs fails (made on the host, before the call is issued): no token of any request is lost."""
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_fork_order import make, rows

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def books(p, nb):
    return p.free_queue().tolist(), [p.refcount(b) for b in range(nb)], [p.info(r)[1]["blocks"].tolist() for r in (1, 2)], [p.info(r)[1]["n_tokens"] for r in (1, 2)]


def test_a_shrink_in_a_full_pool_happens_or_changes_nothing():
    """The copy goes into a block of the request's own tail.  What fails before it leaves all 80 tokens; behind it the shrink stands."""
    n, outcomes = 1, set()
    while True:
        p, dev, _ = make(5)
        with p:
            assert p.admit(1, 32)[0] == p.fork(2, 1, 32)[0] == p.resize(2, 80)[0] == kvr.OK
            torch.cuda.synchronize()
            was1, was2, before = rows(p, dev, 5, 1), rows(p, dev, 5, 2), books(p, 5)
            assert p.free_queue().size == 0 and p.test_fail_nth(kvr.FAIL_CUDA, n) == kvr.OK
            st, table = p.resize(2, 20)
            reached = p.test_points(kvr.FAIL_CUDA) >= n
            p.test_fail_nth(kvr.FAIL_CUDA, 0)
            torch.cuda.synchronize()
            assert torch.equal(rows(p, dev, 5, 1), was1)
            if st == kvr.OK:
                assert table.tolist() == [0, 2] and p.free_queue().tolist() == [3, 4] and [p.refcount(b) for b in range(3)] == [2, 1, 1]
                assert p.suspend_to_host([2])[0] == kvr.OK and p.resume_from_host([2], kvr.SYNC)[0] == kvr.OK
                assert torch.equal(rows(p, dev, 5, 2), was2[:, :, :20])
            else:
                assert st == kvr.ERR_CUDA and books(p, 5) == before and torch.equal(rows(p, dev, 5, 2), was2), n
            outcomes.add((reached, st))
        if not reached:
            break
        n += 1
    assert n > 3 and (False, kvr.OK) in outcomes and (True, kvr.ERR_CUDA) in outcomes


def test_a_growth_that_cannot_be_ordered_behind_a_copy_changes_nothing():
    late, n = torch.cuda.Stream(), 1
    while True:
        p, dev, _ = make(5)
        with p:
            assert p.admit(1, 20)[0] == p.admit(2, 20)[0] == kvr.OK
            torch.cuda.synchronize()
            with torch.cuda.stream(late):
                torch.cuda._sleep(40_000_000)
            assert p.fork(3, 1, 20, stream=late.cuda_stream)[0] == p.release(3) == kvr.OK
            before = books(p, 5)
            assert p.test_fail_nth(kvr.FAIL_CUDA, n) == kvr.OK
            st, table = p.resize(2, 48)
            reached = p.test_points(kvr.FAIL_CUDA) >= n
            p.test_fail_nth(kvr.FAIL_CUDA, 0)
            torch.cuda.synchronize()
            if not reached:
                assert st == kvr.OK and table.tolist() == [2, 3, 4]
                break
            assert st == kvr.ERR_CUDA and books(p, 5) == before
            n += 1
    assert n > 1
