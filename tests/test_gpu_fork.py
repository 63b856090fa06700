"""Fork, resize and compact with bytes: rows that are copied, and the order between these copies and the pool's own moves."""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

GEOM, NB, BS = (3, 2, 64, 2, 16), 64, 16


def make(layout=0, fmt_geom=GEOM, nb=NB, **kw):
    L, H, D, e, bs = fmt_geom
    dev = torch.zeros(2 * L * nb * bs * H * D * e, dtype=torch.uint8, device="cuda")
    p = kvr.Pool(*fmt_geom, nb, 1 << 28, initial_free_order=np.random.default_rng(3).permutation(nb).astype(np.int32), device_pool=dev.data_ptr(), layout=layout, **kw)
    return p, dev


def tiles(dev, layout, geom=GEOM, nb=NB):
    """[layers, 2, blocks, block_size, row] as a view."""
    L, bs = geom[0], geom[4]
    return dev.view(L, 2, nb, bs, -1) if layout == 0 else dev.view(nb, L, 2, bs, -1).permute(1, 2, 0, 3, 4)


def tokens(p, dev, layout, rid, n=None):
    """A request's rows, [layers, 2, tokens, row]."""
    d = p.info(rid)[1]
    t = tiles(dev, layout)[:, :, torch.from_numpy(d["blocks"]).long().cuda()]
    return t.reshape(t.shape[0], 2, -1, t.shape[-1])[:, :, :d["n_tokens"] if n is None else n].clone()


@pytest.mark.parametrize("layout", [0, 1])
def test_a_fork_holds_the_donors_tokens_and_either_goes_on(layout):
    p, dev = make(layout)
    with p:
        assert p.admit(1, 71)[0] == kvr.OK
        dev.random_(0, 256)
        was = tokens(p, dev, layout, 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        assert p.fork(2, 1, 71, stream=side.cuda_stream)[0] == p.fork(3, 1, 64, stream=side.cuda_stream)[0] == p.fork(4, 1, 5, stream=side.cuda_stream)[0] == kvr.OK
        side.synchronize()
        for rid, n in ((2, 71), (3, 64), (4, 5)):
            assert torch.equal(tokens(p, dev, layout, rid), was[:, :, :n])
        # the donor and the fork write their next token into blocks of their own
        for rid, value in ((1, 1), (2, 2)):
            assert p.resize(rid, 72)[0] == kvr.OK
            b = int(p.info(rid)[1]["blocks"][-1])
            tiles(dev, layout)[:, :, b, 71 % BS] = value
        torch.cuda.synchronize()
        assert torch.equal(tokens(p, dev, layout, 1, 71), was) and torch.equal(tokens(p, dev, layout, 2, 71), was)
        assert (tokens(p, dev, layout, 1)[:, :, 71] == 1).all() and (tokens(p, dev, layout, 2)[:, :, 71] == 2).all()
        # drafted tokens that were not accepted: back into a block that others refer to
        assert p.resize(1, 50)[0] == kvr.OK
        torch.cuda.synchronize()
        assert torch.equal(tokens(p, dev, layout, 1), was[:, :, :50]) and torch.equal(tokens(p, dev, layout, 3), was[:, :, :64])
        tiles(dev, layout)[:, :, int(p.info(1)[1]["blocks"][-1]), 50 % BS] = 9
        torch.cuda.synchronize()
        assert torch.equal(tokens(p, dev, layout, 3), was[:, :, :64])


@pytest.mark.parametrize("layout", [0, 1])
def test_compaction_moves_bytes_and_tables(layout):
    p, dev = make(layout)
    with p:
        rng = np.random.default_rng(layout)
        for rid in range(9):
            assert p.admit(rid, int(rng.integers(1, 90)))[0] == kvr.OK
        dev.random_(0, 256)
        assert p.fork(20, 3, p.info(3)[1]["n_tokens"])[0] == kvr.OK
        for rid in (0, 4, 5):
            assert p.release(rid) == kvr.OK
        alive = [1, 2, 3, 6, 7, 8, 20]
        was = {r: tokens(p, dev, layout, r) for r in alive}
        assert p.suspend_to_host([20])[0] == kvr.OK                              # in flight; keeps its prefix
        st, moves = p.compact(3)
        assert st == kvr.OK and len(moves) == 3
        st, more = p.compact()
        torch.cuda.synchronize()
        used = [b for b in range(NB) if p.refcount(b)]
        assert st == kvr.OK and len(more) > 0 and used == list(range(len(used)))
        assert p.compact()[1].size == 0
        for r in alive[:-1]:
            assert torch.equal(tokens(p, dev, layout, r), was[r])
        assert p.resume_from_host([20], kvr.SYNC)[0] == kvr.OK and torch.equal(tokens(p, dev, layout, 20), was[20])


def test_compaction_of_more_pairs_than_one_launch_takes():
    geom = (1, 1, 16, 2, 1)                                                      # a block is one token of 32 bytes
    p, dev = make(0, geom, 8192)
    with p:
        for rid in range(6000):
            assert p.admit(rid, 1)[0] == kvr.OK
        dev.random_(0, 256)
        t = tiles(dev, 0, geom, 8192)
        keep = list(range(0, 6000, 2))
        was = torch.stack([t[:, :, int(p.info(r)[1]["blocks"][0])] for r in keep])
        for rid in range(1, 6000, 2):
            assert p.release(rid) == kvr.OK
        st, moves = p.compact()
        torch.cuda.synchronize()
        assert st == kvr.OK and len(moves) > 1024 and not {a for a, _ in moves.tolist()} & {b for _, b in moves.tolist()}
        assert torch.equal(torch.stack([t[:, :, int(p.info(r)[1]["blocks"][0])] for r in keep]), was)


def test_moves_come_behind_the_copies_and_copies_behind_the_moves():
    """Nothing here waits between the calls: a fork of a resuming donor, into blocks that a suspend still reads; suspends of what was just
    copied, behind work that keeps the caller's stream busy."""
    p, dev = make()
    side, heavy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    with p:
        for turn in range(20):
            assert p.admit(1, 500)[0] == p.admit(2, 300)[0] == kvr.OK
            torch.cuda.synchronize()
            dev.random_(0, 256)
            torch.cuda.synchronize()
            was1, was2 = tokens(p, dev, 0, 1), tokens(p, dev, 0, 2)
            assert p.suspend_to_host([1])[0] == kvr.OK
            assert p.resume_from_host([1])[0] == kvr.OK
            with torch.cuda.stream(side):
                heavy @ heavy                                                    # the copies queue behind this
            assert p.fork(3, 1, 499, stream=side.cuda_stream)[0] == kvr.OK
            assert p.resize(2, 211, stream=side.cuda_stream)[0] == kvr.OK
            assert p.suspend_to_host([3, 2])[0] == kvr.OK                        # reads what the copy writes
            assert p.release(1) == kvr.OK
            assert p.resume_from_host([3, 2], kvr.SYNC)[0] == kvr.OK
            side.synchronize()
            assert torch.equal(tokens(p, dev, 0, 3), was1[:, :, :499]) and torch.equal(tokens(p, dev, 0, 2), was2[:, :, :211])
            assert p.release(3) == p.release(2) == kvr.OK


def test_a_stream_under_capture_is_refused_and_a_failed_call_changes_nothing():
    p, dev = make()
    with p:
        assert p.admit(1, 50)[0] == kvr.OK and p.admit(2, 60)[0] == kvr.OK
        graph, x = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
        with torch.cuda.graph(graph):
            x += 1
            s = torch.cuda.current_stream().cuda_stream
            assert p.fork(3, 1, 50, stream=s)[0] == p.resize(1, 20, stream=s)[0] == p.compact(stream=s)[0] == kvr.ERR_INVALID_ARG
        graph.replay()
        torch.cuda.synchronize()
        assert (x == 1).all()
        dev.random_(0, 256)
        assert p.fork(4, 2, 48)[0] == kvr.OK and p.release(1) == kvr.OK
        before = (p.free_queue().tolist(), p.info(2)[1]["blocks"].tolist(), [p.refcount(b) for b in range(NB)], tokens(p, dev, 0, 2))
        for call in (lambda: p.fork(3, 2, 59), lambda: p.resize(2, 41), lambda: p.resize(2, 3), lambda: p.compact()):
            n = 1
            while True:
                assert p.test_fail_nth(kvr.FAIL_CUDA, n) == kvr.OK
                st, table = call()
                if p.test_points(kvr.FAIL_CUDA) < n:
                    break
                assert st == kvr.ERR_CUDA, n
                after = (p.free_queue().tolist(), p.info(2)[1]["blocks"].tolist(), [p.refcount(b) for b in range(NB)])
                assert after == before[:3] and torch.equal(tokens(p, dev, 0, 2), before[3]) and p.info(3)[0] == kvr.ERR_UNKNOWN_REQUEST
                n += 1
            assert n > 3
            p.test_fail_nth(kvr.FAIL_CUDA, 0)
            # take the call that went through back
            if st == kvr.OK and p.info(3)[0] == kvr.OK:
                assert p.release(3) == kvr.OK
            before = (p.free_queue().tolist(), p.info(2)[1]["blocks"].tolist(), [p.refcount(b) for b in range(NB)], tokens(p, dev, 0, 2))
