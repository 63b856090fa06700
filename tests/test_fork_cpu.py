"""Fork, resize and compact: the books of a metadata-only pool against a plain model, what they refuse, and a state that a failure leaves as it was."""
import collections

import numpy as np
import pytest

from paper_2608_30830_b200 import kvr

BS = 4


class Model:
    """Tables, reference counts and the free queue as the header has them."""

    def __init__(self, order):
        self.free, self.reqs, self.n = collections.deque(order), {}, len(order)

    def refs(self, b):
        return sum(r["blocks"].count(b) for r in self.reqs.values())

    def drop(self, blocks, rid):
        for b in blocks:
            self.reqs[rid]["blocks"].remove(b)
            if self.refs(b) == 0:
                self.free.append(b)

    def admit(self, rid, n):
        nb = -(-n // BS)
        if rid in self.reqs and self.reqs[rid]["state"] != kvr.EXPIRED:
            return kvr.ERR_BAD_STATE
        if nb > len(self.free):
            return kvr.HBM_FULL
        self.reqs[rid] = dict(n=n, shared=0, state=kvr.ACTIVE, blocks=[self.free.popleft() for _ in range(nb)])
        return kvr.OK

    def fork(self, rid, donor, n):
        if donor == rid:
            return kvr.ERR_INVALID_ARG
        if donor not in self.reqs:
            return kvr.ERR_UNKNOWN_REQUEST
        d = self.reqs[donor]
        if d["state"] not in (kvr.ACTIVE, kvr.RETAINED):
            return kvr.ERR_BAD_STATE
        if n > d["n"]:
            return kvr.ERR_INVALID_ARG
        if rid in self.reqs and self.reqs[rid]["state"] != kvr.EXPIRED:
            return kvr.ERR_BAD_STATE
        if n % BS and not self.free:
            return kvr.HBM_FULL
        full = n // BS
        self.reqs[rid] = dict(n=n, shared=full, state=kvr.ACTIVE, blocks=d["blocks"][:full] + ([self.free.popleft()] if n % BS else []))
        return kvr.OK

    def resize(self, rid, n):
        if rid not in self.reqs:
            return kvr.ERR_UNKNOWN_REQUEST
        r, nb = self.reqs[rid], -(-n // BS)
        if r["state"] != kvr.ACTIVE:
            return kvr.ERR_BAD_STATE
        if nb - len(r["blocks"]) > len(self.free):
            return kvr.HBM_FULL
        if nb > len(r["blocks"]):
            r["blocks"] += [self.free.popleft() for _ in range(nb - len(r["blocks"]))]
        else:
            tail = r["blocks"][nb:]
            if n % BS and self.refs(r["blocks"][nb - 1]) > 1:
                own = self.free.popleft() if self.free else next((b for b in tail if self.refs(b) == 1), None)
                if own is None:
                    return kvr.HBM_FULL
                if own in tail:
                    tail.remove(own)
                    r["blocks"].remove(own)
                old, r["blocks"][nb - 1] = r["blocks"][nb - 1], own
                assert self.refs(old) > 0
            for b in tail:
                r["blocks"].remove(b)
                if self.refs(b) == 0:
                    self.free.append(b)
        r["n"], r["shared"] = n, min(r["shared"], n // BS)
        return kvr.OK

    def compact(self, most):
        moves = []
        while len(moves) < most:
            used = [b for b in range(self.n) if b not in self.free]
            lo = min(self.free, default=self.n)
            if not used or lo > used[-1]:
                break
            moves.append([used[-1], lo])
            for r in self.reqs.values():
                r["blocks"] = [lo if b == used[-1] else b for b in r["blocks"]]
            self.free.remove(lo)
            self.free.append(used[-1])
        return moves

    def suspend(self, rid):
        r = self.reqs.get(rid)
        if r is None:
            return kvr.ERR_UNKNOWN_REQUEST
        if r["state"] not in (kvr.ACTIVE, kvr.RETAINED):
            return kvr.ERR_BAD_STATE
        r["state"] = kvr.HOST
        gone, r["blocks"] = r["blocks"][r["shared"]:], r["blocks"][:r["shared"]]
        for b in gone:
            if self.refs(b) == 0:
                self.free.append(b)
        return kvr.OK

    def resume(self, rid):
        r = self.reqs.get(rid)
        if r is None:
            return kvr.ERR_UNKNOWN_REQUEST
        if r["state"] != kvr.HOST:
            return kvr.ERR_BAD_STATE
        need = -(-r["n"] // BS) - r["shared"]
        if need > len(self.free):
            return kvr.HBM_FULL
        r["blocks"] += [self.free.popleft() for _ in range(need)]
        r["state"] = kvr.ACTIVE
        return kvr.OK

    def release(self, rid):
        if rid not in self.reqs:
            return kvr.ERR_UNKNOWN_REQUEST
        blocks = self.reqs[rid]["blocks"]
        self.reqs[rid]["blocks"] = []
        for i, b in enumerate(blocks):
            if self.refs(b) == 0 and b not in blocks[i + 1:]:
                self.free.append(b)
        del self.reqs[rid]
        return kvr.OK


def pool(nb, order=None):
    return kvr.Pool(2, 2, 8, 2, BS, nb, 1 << 24, flags=kvr.METADATA_ONLY, initial_free_order=order)


def same(p, m):
    assert p.free_queue().tolist() == list(m.free)
    for b in range(m.n):
        assert p.refcount(b) == m.refs(b)
    for rid, r in m.reqs.items():
        st, d = p.info(rid)
        assert st == kvr.OK and d["state"] == r["state"] and d["n_tokens"] == r["n"] and d["nb"] == -(-r["n"] // BS)
        assert d["image_bytes"] == (r["n"] - r["shared"] * BS) * kvr.bytes_per_token(2, 2, 8, 2, BS) if r["state"] != kvr.EXPIRED else True
        assert p.sharing(rid)[1].tolist() == r["blocks"][:r["shared"]]
        if r["state"] == kvr.ACTIVE:
            assert d["blocks"].tolist() == r["blocks"]


@pytest.mark.parametrize("seed", range(6))
def test_any_run_of_calls_keeps_the_books_of_the_model(seed):
    rng = np.random.default_rng(seed)
    nb = int(rng.integers(6, 16))
    order = rng.permutation(nb).astype(np.int32)
    m, seen = Model(order.tolist()), set()
    with pool(nb, order) as p:
        for _ in range(400):
            rid, other, n = int(rng.integers(0, 6)), int(rng.integers(0, 6)), int(rng.integers(0, 10 * BS))
            if other in m.reqs and rng.random() < 0.7:
                n = int(rng.integers(0, m.reqs[other]["n"] + 2))
            what = rng.choice(["admit", "fork", "fork", "resize", "resize", "resize", "compact", "suspend", "resume", "release"])
            if what == "admit":
                want, got = m.admit(rid, n), p.admit(rid, n)[0]
            elif what == "fork":
                want, (got, table) = m.fork(rid, other, n), p.fork(rid, other, n)
                assert table is None or table.tolist() == m.reqs[rid]["blocks"]
            elif what == "resize":
                want, (got, table) = m.resize(rid, n), p.resize(rid, n)
                assert table is None or table.tolist() == m.reqs[rid]["blocks"]
            elif what == "compact":
                most = int(rng.integers(0, 8))
                st, moves = p.compact(most)
                want, got = (kvr.OK, m.compact(most)), (st, moves.tolist())
            elif what == "release":
                want, got = m.release(rid), p.release(rid)
            else:
                want = (m.suspend if what == "suspend" else m.resume)(rid)
                got = (p.suspend_to_host if what == "suspend" else p.resume_from_host)([rid])[1][0]
            assert got == want, (what, rid, other, n)
            seen.add((what, want if isinstance(want, int) else kvr.OK))
            same(p, m)
    assert {("fork", kvr.OK), ("resize", kvr.OK), ("compact", kvr.OK)} <= seen


def test_a_shared_block_is_not_written_on_after_a_shrink():
    with pool(8) as p:
        assert p.admit(1, 3 * BS)[0] == p.fork(2, 1, 3 * BS)[0] == kvr.OK
        st, table = p.resize(1, 2 * BS + 1)                       # its third block is the fork's too
        assert st == kvr.OK and table.tolist() == [0, 1, 3] and p.info(2)[1]["blocks"].tolist() == [0, 1, 2]
        assert [p.refcount(b) for b in range(4)] == [2, 2, 1, 1]
        assert p.resize(1, 2 * BS + 2)[1].tolist() == [0, 1, 3]   # its own now
        assert p.resize(2, BS)[1].tolist() == [0] and p.free_queue().tolist() == [4, 5, 6, 7, 2]
        assert p.sharing(2)[1].tolist() == [0]
        assert p.resize(2, 0)[0] == kvr.OK and p.refcount(0) == 1 and p.info(2)[1]["image_bytes"] == 0


def test_a_copy_goes_into_the_requests_own_tail_where_the_pool_is_full():
    with pool(5) as p:
        assert p.admit(1, 2 * BS)[0] == p.fork(2, 1, 2 * BS)[0] == kvr.OK
        assert p.resize(2, 5 * BS)[1].tolist() == [0, 1, 2, 3, 4]
        assert p.resize(1, BS + 1)[0] == kvr.HBM_FULL             # nowhere to put the copy
        assert p.info(1)[1]["blocks"].tolist() == [0, 1] and p.info(1)[1]["n_tokens"] == 2 * BS
        assert p.resize(2, BS + 1)[1].tolist() == [0, 2] and p.free_queue().tolist() == [3, 4]
        assert [p.refcount(b) for b in range(5)] == [2, 1, 1, 0, 0]


def test_refusals():
    L = kvr.lib()
    with pool(4) as p:
        assert p.admit(1, 5)[0] == kvr.OK
        assert p.fork(2, 1, -1)[0] == p.fork(1, 1, 3)[0] == p.fork(2, 1, 6)[0] == kvr.ERR_INVALID_ARG and kvr.last_error()
        assert p.fork(2, 7, 1)[0] == p.resize(7, 1)[0] == kvr.ERR_UNKNOWN_REQUEST
        assert p.resize(1, -1)[0] == kvr.ERR_INVALID_ARG and p.resize(1, 17)[0] == kvr.HBM_FULL and L.kvr_request_resize(p._h, 1, 1 << 60, None, 0, None) == kvr.HBM_FULL
        assert p.fork(2, 1, 5)[0] == kvr.OK and p.fork(2, 1, 5)[0] == kvr.ERR_BAD_STATE
        out = np.zeros(1, dtype=np.int32)
        assert L.kvr_request_fork(p._h, 3, 1, 5, kvr._i32p(out), 1, None) == L.kvr_request_resize(p._h, 1, 5, kvr._i32p(out), 1, None) == kvr.ERR_INVALID_ARG
        assert p.compact(-1)[0] == kvr.ERR_INVALID_ARG and p.compact(0)[0] == kvr.OK
        for fn, args in ((L.kvr_request_fork, (2, 1, 0, None, 0, None)), (L.kvr_request_resize, (1, 0, None, 0, None)), (L.kvr_pool_compact, (1, None, None, None))):
            assert fn(None, *args) == kvr.ERR_INVALID_ARG
        assert p.suspend_to_host([1])[0] == kvr.OK
        assert p.fork(3, 1, 1)[0] == p.resize(1, 1)[0] == kvr.ERR_BAD_STATE
        assert p.expire([2])[0] == kvr.OK and p.resize(2, 1)[0] == kvr.ERR_BAD_STATE
        assert p.resume_from_host([1])[0] == kvr.OK and p.retain_in_hbm([1])[0] == kvr.OK
        assert p.resize(1, 1)[0] == kvr.ERR_BAD_STATE and p.fork(2, 1, 5)[0] == kvr.OK          # an expired id may come back
        assert L.kvr_request_fork(p._h, 9, 1, 0, None, 0, None) == kvr.OK and p.info(9)[1]["nb"] == 0
