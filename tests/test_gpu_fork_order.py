"""Fork, resize and compact against work that is still under way: a pool's gathers and scatters, and copies on other streams, all made late
by a stream that is busy.  Nothing waits between the calls but the calls themselves."""
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_fork import GEOM, tiles

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

ROUTES = {"staged": kvr.ROUTE_STAGED, "mapped": kvr.ROUTE_MAPPED, "dma2d": kvr.ROUTE_DMA2D}


def make(nb, route="staged"):
    """A pool in the order of its ids, its memory full of random bytes, and its four streams."""
    L, H, D, e, bs = GEOM
    dev = torch.randint(0, 256, (2 * L * nb * bs * H * D * e,), dtype=torch.uint8, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(4)]
    p = kvr.Pool(*GEOM, nb, 1 << 26, device_pool=dev.data_ptr(), route=ROUTES[route], chunk_bytes=1 << 20, staging_slots=4, streams=[s.cuda_stream for s in streams])
    torch.cuda.synchronize()
    return p, dev, streams


def busy(stream, cycles=40_000_000):
    """About 20 ms of work."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(cycles)


def write(dev, nb, blocks, value, stream, rows=slice(None)):
    with torch.cuda.stream(stream):
        for b in blocks:
            tiles(dev, 0, GEOM, nb)[:, :, int(b), rows] = value


@pytest.fixture(autouse=True, scope="module")
def loaded():
    """Every kernel has run once: the first launch of one waits for the device."""
    for route in ROUTES:
        p, dev, streams = make(8, route)
        with p:
            assert p.admit(1, 20)[0] == p.fork(2, 1, 20)[0] == p.suspend_to_host([1])[0] == p.resume_from_host([1], kvr.SYNC)[0] == kvr.OK
            write(dev, 8, [7], 1, streams[0])
            rows(p, dev, 8, 1)
            busy(streams[0])
            torch.cuda.synchronize()


def reader(streams, route):
    """The stream that reads the blocks of a suspend."""
    return streams[1 if route == "dma2d" else 0]


def rows(p, dev, nb, rid, n=None):
    """A request's rows, [layers, 2, tokens, row]."""
    d = p.info(rid)[1]
    t = tiles(dev, 0, GEOM, nb)[:, :, torch.from_numpy(d["blocks"]).long().cuda()]
    return t.reshape(t.shape[0], 2, -1, t.shape[-1])[:, :, :d["n_tokens"] if n is None else n].clone()


@pytest.mark.parametrize("route", ROUTES)
def test_a_shrink_waits_for_the_suspend_that_still_reads_the_block(route):
    p, dev, streams = make(8, route)
    with p:
        assert p.admit(1, 32)[0] == p.fork(2, 1, 32)[0] == kvr.OK
        was = rows(p, dev, 8, 1)
        torch.cuda.synchronize()
        busy(reader(streams, route))
        assert p.suspend_to_host([1])[0] == kvr.OK
        st, table = p.resize(2, 20)                          # block 1 is its own now, and will be written on
        assert st == kvr.OK and table.tolist() == [0, 1] and p.refcount(1) == 1
        tiles(dev, 0, GEOM, 8)[:, :, 1, 4:] = 7
        torch.cuda.synchronize()
        assert p.resume_from_host([1], kvr.SYNC)[0] == kvr.OK
        assert torch.equal(rows(p, dev, 8, 1), was) and torch.equal(rows(p, dev, 8, 2), was[:, :, :20])


@pytest.mark.parametrize("route", ROUTES)
def test_a_copy_into_the_requests_own_tail_waits_for_the_suspend_that_still_reads_it(route):
    p, dev, streams = make(5, route)
    with p:
        assert p.admit(1, 80)[0] == p.fork(2, 1, 80)[0] == p.fork(3, 1, 32)[0] == kvr.OK
        was = rows(p, dev, 5, 1)
        torch.cuda.synchronize()
        busy(reader(streams, route))
        assert p.suspend_to_host([1])[0] == kvr.OK
        st, table = p.resize(2, 20)                          # block 1 is request 3's too, and no block is free
        assert st == kvr.OK and table.tolist() == [0, 2]
        torch.cuda.synchronize()
        assert torch.equal(rows(p, dev, 5, 2), was[:, :, :20]) and torch.equal(rows(p, dev, 5, 3), was[:, :, :32])
        assert p.release(2) == p.release(3) == kvr.OK
        assert p.resume_from_host([1], kvr.SYNC)[0] == kvr.OK and torch.equal(rows(p, dev, 5, 1), was)


# ---- copies that are late: their stream is busy, and whoever takes one of their blocks comes from elsewhere

def test_admit_waits_for_a_copy_that_reads_or_writes_its_blocks():
    p, dev, _ = make(4)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        for call in ("admit", "admit_into", "admit_sharing", "admit_sharing_into"):
            for gone in (1, 2):                              # the source's owner, the destination's
                assert p.admit(1, 20)[0] == kvr.OK
                was = rows(p, dev, 4, 1)
                torch.cuda.synchronize()
                busy(late)
                assert p.fork(2, 1, 20, stream=late.cuda_stream)[0] == kvr.OK
                last = int(p.info(gone)[1]["blocks"][1])
                assert p.release(gone) == kvr.OK
                free = p.free_queue()
                assert last in free
                if call == "admit":
                    assert p.admit(3, 32)[0] == kvr.OK
                elif call == "admit_into":
                    assert p.admit_into(3, 32, free) == kvr.OK
                elif call == "admit_sharing":
                    assert p.admit_sharing(3, 48, 3 - gone, 1)[0] == kvr.OK
                else:
                    assert p.admit_sharing_into(3, 48, 3 - gone, 1, free) == kvr.OK
                write(dev, 4, free, 9, other)
                torch.cuda.synchronize()
                assert torch.equal(rows(p, dev, 4, 3 - gone), was)
                assert all((tiles(dev, 0, GEOM, 4)[:, :, int(b)] == 9).all() for b in free)
                assert p.release(3) == p.release(3 - gone) == kvr.OK


def test_copies_on_two_streams_that_use_one_block_come_one_after_the_other():
    p, dev, _ = make(5)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        assert p.admit(1, 20)[0] == p.admit(5, 20)[0] == kvr.OK
        was = rows(p, dev, 5, 1), rows(p, dev, 5, 5)
        torch.cuda.synchronize()
        busy(late)
        assert p.fork(2, 1, 20, stream=late.cuda_stream)[1].tolist() == [0, 4]
        assert p.release(2) == kvr.OK
        assert p.fork(6, 5, 20, stream=other.cuda_stream)[1].tolist() == [2, 4]                  # the same destination
        assert p.fork(7, 6, 16, stream=late.cuda_stream)[0] == kvr.OK
        torch.cuda.synchronize()
        assert torch.equal(rows(p, dev, 5, 6), was[1]) and torch.equal(rows(p, dev, 5, 5), was[1]) and torch.equal(rows(p, dev, 5, 1), was[0])
        # a fork of what is still being copied
        assert p.release(6) == p.release(7) == p.release(1) == kvr.OK
        torch.cuda.synchronize()
        busy(late)
        assert p.fork(8, 5, 20, stream=late.cuda_stream)[0] == kvr.OK
        assert p.fork(9, 8, 19, stream=other.cuda_stream)[0] == kvr.OK
        torch.cuda.synchronize()
        assert torch.equal(rows(p, dev, 5, 8), was[1]) and torch.equal(rows(p, dev, 5, 9), was[1][:, :, :19])


def test_a_growing_request_comes_behind_a_late_copy_into_its_new_block():
    p, dev, _ = make(5)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        assert p.admit(1, 20)[0] == p.admit(5, 20)[0] == kvr.OK
        torch.cuda.synchronize()
        busy(late)
        assert p.fork(2, 1, 20, stream=late.cuda_stream)[0] == p.release(2) == kvr.OK
        assert p.resize(5, 48, stream=other.cuda_stream)[1].tolist() == [2, 3, 4]
        write(dev, 5, [4], 9, other)
        torch.cuda.synchronize()
        assert (tiles(dev, 0, GEOM, 5)[:, :, 4] == 9).all()


def test_a_shrink_comes_behind_a_late_copy_of_the_rows_it_takes_back():
    p, dev, _ = make(5)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        assert p.admit(1, 20)[0] == kvr.OK
        was = rows(p, dev, 5, 1)
        torch.cuda.synchronize()
        busy(late)
        assert p.fork(2, 1, 20, stream=late.cuda_stream)[0] == kvr.OK
        assert p.resize(1, 17, stream=other.cuda_stream)[1].tolist() == [0, 1]
        write(dev, 5, [1], 9, other, slice(1, None))
        torch.cuda.synchronize()
        assert torch.equal(rows(p, dev, 5, 2), was) and torch.equal(rows(p, dev, 5, 1), was[:, :, :17])


def test_a_block_that_a_shrink_let_go_is_copied_into_behind_the_work_on_it():
    p, dev, _ = make(5)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        assert p.admit(1, 20)[0] == p.admit(2, 48)[0] == kvr.OK
        was = rows(p, dev, 5, 1), rows(p, dev, 5, 2)
        torch.cuda.synchronize()
        busy(late)
        with torch.cuda.stream(late):
            seen = rows(p, dev, 5, 2)                        # the caller's own reading, late
        assert p.resize(2, 32, stream=late.cuda_stream)[0] == kvr.OK
        assert p.fork(3, 1, 20, stream=other.cuda_stream)[1].tolist() == [0, 4]
        torch.cuda.synchronize()
        assert torch.equal(seen, was[1]) and torch.equal(rows(p, dev, 5, 3), was[0])


def test_blocks_that_a_compaction_moved_away_from_are_handed_out_behind_it():
    p, dev, _ = make(3)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        assert p.admit(1, 16)[0] == p.admit(2, 16)[0] == kvr.OK
        was = rows(p, dev, 3, 2)
        torch.cuda.synchronize()
        assert p.release(1) == kvr.OK
        busy(late)
        assert p.compact(stream=late.cuda_stream)[1].tolist() == [[1, 0]]
        assert p.admit(3, 32)[1].tolist() == [2, 1]
        write(dev, 3, [1, 2], 9, other)
        torch.cuda.synchronize()
        assert torch.equal(rows(p, dev, 3, 2), was)


def test_a_compaction_comes_behind_late_copies_on_other_streams():
    p, dev, _ = make(40)
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    with p:
        for many in (1, 30):                                 # a few pairs, and more than are looked at one by one
            for rid in range(many):
                assert p.admit(100 + rid, 1)[0] == kvr.OK
            assert p.admit(1, 20)[0] == kvr.OK
            was = rows(p, dev, 40, 1)
            torch.cuda.synchronize()
            busy(late)
            assert p.fork(2, 1, 20, stream=late.cuda_stream)[0] == kvr.OK
            for rid in range(many):
                assert p.release(100 + rid) == kvr.OK
            assert len(p.compact(stream=other.cuda_stream)[1]) > 0
            torch.cuda.synchronize()
            assert torch.equal(rows(p, dev, 40, 1), was) and torch.equal(rows(p, dev, 40, 2), was)
            assert p.release(1) == p.release(2) == kvr.OK


# ---- resumes that are late: the stream that writes the blocks is busy

@pytest.mark.parametrize("what", ["resume", "import"])
@pytest.mark.parametrize("route", ROUTES)
def test_a_copy_out_of_a_prefix_that_another_requests_move_still_fills(route, what):
    p, dev, streams = make(16, route)
    side = torch.cuda.Stream()
    with p:
        assert p.admit(1, 40)[0] == kvr.OK
        was = rows(p, dev, 16, 1)
        buffer = torch.zeros(40 * 2 * GEOM[0] * was.shape[-1] + 256, dtype=torch.uint8, device="cuda")
        if what == "import":
            assert p.export_to_device([1], buffer.data_ptr(), buffer.numel(), kvr.SYNC)[0] == kvr.OK
        else:
            assert p.suspend_to_host([1], kvr.SYNC)[0] == kvr.OK
        dev.random_(0, 256)
        torch.cuda.synchronize()
        busy(streams[2 if route == "dma2d" and what == "resume" else 3])
        if what == "import":
            assert p.import_from_device([1], buffer.data_ptr(), buffer.numel())[0] == kvr.OK
        else:
            assert p.resume_from_host([1])[0] == kvr.OK
        assert p.admit_sharing(2, 32, 1, 2)[0] == p.admit_sharing(5, 32, 1, 2)[0] == kvr.OK
        assert p.fork(3, 2, 21, stream=side.cuda_stream)[0] == p.fork(4, 2, 32, stream=side.cuda_stream)[0] == kvr.OK
        with torch.cuda.stream(side):
            shared = rows(p, dev, 16, 4)                     # what a kernel on the fork's stream sees
        assert p.resize(2, 19, stream=side.cuda_stream)[0] == kvr.OK
        table = p.resize(5, 30, stream=torch.cuda.Stream().cuda_stream)[1]
        assert table[1] != p.info(1)[1]["blocks"][1]
        torch.cuda.synchronize()
        for rid, n in ((1, 40), (2, 19), (3, 21), (4, 32), (5, 30)):
            assert torch.equal(rows(p, dev, 16, rid), was[:, :, :n]), rid
        assert torch.equal(shared, was[:, :, :32])


def test_no_stream_is_the_current_one():
    """As for Cache: what the current stream is about to write is what a fork, a shrink and a compaction copy."""
    p, dev, _ = make(8)
    side = torch.cuda.Stream()
    with p:
        assert p.admit(9, 16)[0] == p.admit(1, 48)[0] == p.fork(5, 1, 48)[0] == kvr.OK
        torch.cuda.synchronize()
        busy(side)
        write(dev, 8, [1, 2, 3], 9, side)
        with torch.cuda.stream(side):
            assert p.fork(2, 1, 40)[0] == kvr.OK
            assert p.resize(5, 20)[0] == kvr.OK
            assert p.release(9) == kvr.OK
            assert len(p.compact()[1]) == 1
        torch.cuda.synchronize()
        for rid in (1, 2, 5):
            assert (rows(p, dev, 8, rid) == 9).all(), rid


def test_a_current_stream_under_capture_is_refused():
    p, dev, _ = make(8)
    with p:
        assert p.admit(1, 20)[0] == kvr.OK
        graph, x = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
        with torch.cuda.graph(graph):
            x += 1
            assert p.fork(3, 1, 20)[0] == p.resize(1, 5)[0] == p.compact()[0] == kvr.ERR_INVALID_ARG
        graph.replay()
        torch.cuda.synchronize()
        assert (x == 1).all() and p.info(1)[1]["n_tokens"] == 20


def test_many_copies_under_way_on_several_streams():
    """More than are kept before those that are through are looked for; then all of their blocks change hands."""
    p, dev, _ = make(200)
    streams = [torch.cuda.Stream() for _ in range(20)]       # more than one look tells apart
    with p:
        assert p.admit(1, 40)[0] == kvr.OK
        was = rows(p, dev, 200, 1)
        for turn in range(3):
            torch.cuda.synchronize()
            for s in streams[::2]:
                busy(s, 4_000_000)
            for i in range(190):
                assert p.fork(10 + i, 1, 35 + i % 5, stream=streams[(i * 7 + turn) % 20].cuda_stream)[0] == kvr.OK
            if turn == 1:
                torch.cuda.synchronize()
            if turn == 2:
                for i in range(190):
                    assert p.release(10 + i) == kvr.OK
                st, table = p.admit(2, 190 * 16)
                write(dev, 200, table, 9, streams[1])
                torch.cuda.synchronize()
                assert st == kvr.OK and (rows(p, dev, 200, 2) == 9).all() and torch.equal(rows(p, dev, 200, 1), was)
                break
            torch.cuda.synchronize()
            for i in range(190):
                assert torch.equal(rows(p, dev, 200, 10 + i), was[:, :, :35 + i % 5])
                assert p.release(10 + i) == kvr.OK
