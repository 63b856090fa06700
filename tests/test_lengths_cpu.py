"""Lengths near the end of 64 bits: no sum of them with a block's size may wrap.  A metadata-only pool."""
import numpy as np
import pytest

from paper_2608_30830_b200 import kvr

BS = 16
LONG = [2**63 - 1, 2**63 - 2, 2**63 - BS + 1, 2**63 - BS, 2**63 - BS - 1, 2**62, 2**36 + 3, 2**31 * BS]


def pool(nb=4):
    return kvr.Pool(2, 2, 8, 2, BS, nb, 1 << 24, flags=kvr.METADATA_ONLY)


def books(p):
    return p.free_queue().tolist(), [p.refcount(b) for b in range(4)]


@pytest.mark.parametrize("n", LONG)
def test_a_resize_to_more_than_any_pool_holds_changes_nothing(n):
    L = kvr.lib()
    with pool() as p:
        assert p.admit(1, 20)[0] == p.admit(2, 0)[0] == kvr.OK
        was = books(p)
        for rid in (1, 2):
            assert L.kvr_request_resize(p._h, rid, n, None, 0, None) == kvr.HBM_FULL
        assert p.admit(3, 32)[0] == kvr.OK and p.free_queue().size == 0          # the same with nothing free
        full = books(p)
        for rid in (1, 2):
            assert L.kvr_request_resize(p._h, rid, n, None, 0, None) == kvr.HBM_FULL
        out = np.zeros(4, dtype=np.int32)
        assert L.kvr_request_resize(p._h, 1, n, kvr._i32p(out), 4, None) == kvr.ERR_INVALID_ARG
        assert books(p) == full and p.info(1)[1]["n_tokens"] == 20 and p.info(2)[1]["n_tokens"] == 0
        assert p.release(3) == kvr.OK and books(p)[1] == was[1]


@pytest.mark.parametrize("n", LONG)
def test_a_request_longer_than_any_pool_is_not_admitted(n):
    L = kvr.lib()
    with pool() as p:
        assert p.admit(1, 40)[0] == kvr.OK
        was = books(p)
        assert L.kvr_request_admit(p._h, 2, n, None, 0) == kvr.HBM_FULL
        assert L.kvr_request_admit_sharing(p._h, 2, n, 1, 2, None, 0) == kvr.HBM_FULL
        ids = np.array([3], dtype=np.int32)
        assert L.kvr_request_admit_into(p._h, 2, n, kvr._i32p(ids), 1) == kvr.ERR_INVALID_ARG
        assert L.kvr_request_admit_sharing_into(p._h, 2, n, 1, 2, kvr._i32p(ids), 1) == kvr.ERR_INVALID_ARG
        for shared, private in ((2**31 - 1, 1), (2**31 - 2, 2)):                  # these add up to the blocks of 2^35 tokens
            assert L.kvr_request_admit_sharing_into(p._h, 2, 2**31 * BS, 1, shared, kvr._i32p(ids), private) == kvr.ERR_INVALID_ARG
        assert L.kvr_request_fork(p._h, 2, 1, n, None, 0, None) == kvr.ERR_INVALID_ARG
        assert books(p) == was and p.info(2)[0] == kvr.ERR_UNKNOWN_REQUEST


@pytest.mark.parametrize("n", [2**64, 2**64 + 5, 2**63, -2**63 - 1])
def test_the_binding_drops_no_bits_of_a_length(n):
    with pool() as p:
        assert p.admit(1, 40)[0] == kvr.OK
        was = books(p)
        for call in (lambda: p.resize(1, n), lambda: p.fork(2, 1, n), lambda: p.compact(n)):
            with pytest.raises(ValueError):
                call()
        assert books(p) == was and p.info(1)[1]["n_tokens"] == 40 and p.info(2)[0] == kvr.ERR_UNKNOWN_REQUEST


def test_the_binding_takes_any_length_that_fits():
    with pool() as p:
        assert p.admit(1, 40)[0] == kvr.OK
        for n in LONG:
            assert p.resize(1, n) == (kvr.HBM_FULL, None) and p.fork(2, 1, n) == (kvr.ERR_INVALID_ARG, None)
        assert p.resize(1, -2**63) == (kvr.ERR_INVALID_ARG, None)
        assert p.admit(2, 10)[0] == p.release(1) == kvr.OK                       # block 3 is in use, 0 to 2 are free
        for most in (-1, -2**31, -2**63):
            assert p.compact(most)[0] == kvr.ERR_INVALID_ARG
        assert p.compact(2**63 - 1)[1].tolist() == [[3, 0]]
