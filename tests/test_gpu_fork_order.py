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


def busy(stream):
    """About 20 ms of work."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(40_000_000)


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
