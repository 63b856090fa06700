"""Runs of fork, resize, compact, admit, suspend and resume on several streams that are busy at random, with the bytes of every request followed
on the host.  The test orders what is the caller's to order (its own writes on one stream before the use of the same tokens on another, and before a suspend); the calls order the rest."""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_fork import GEOM, tiles
from test_gpu_fork_order import busy, loaded, make, rows  # noqa: F401 (loaded: a fixture)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

NB, BS = 24, 16


@pytest.mark.parametrize("route", ["staged", "dma2d"])
@pytest.mark.parametrize("seed", range(5))
def test_any_run_of_calls_on_several_streams_keeps_every_token(seed, route):
    rng = np.random.default_rng(seed)
    p, dev, moves = make(NB, route)
    streams = [torch.cuda.Stream() for _ in range(3)]
    want, owner, state, value, done = {}, {}, {}, 0, {"fork": 0, "compact": 0, "resize": 0, "resume": 0}

    def on_tokens(rid, first, last):
        """The caller writes tokens of a request, on its stream."""
        nonlocal value
        blocks = p.info(rid)[1]["blocks"]
        with torch.cuda.stream(owner[rid]):
            for b in range(first // BS, -(-last // BS)):
                value = value % 250 + 1
                lo, hi = max(first, b * BS), min(last, (b + 1) * BS)
                tiles(dev, 0, GEOM, NB)[:, :, int(blocks[b]), lo - b * BS:hi - b * BS] = value
                want[rid][lo:hi] = value

    def check():
        torch.cuda.synchronize()
        assert p.wait() == kvr.OK
        for rid, s in state.items():
            if s == kvr.ACTIVE:
                got = rows(p, dev, NB, rid)
                assert torch.equal(got, torch.from_numpy(want[rid]).cuda()[None, None, :, None].expand_as(got)), rid

    with p:
        for turn in range(150):
            rid, other, s = int(rng.integers(0, 8)), int(rng.integers(0, 8)), streams[rng.integers(0, 3)]
            if rng.random() < 0.3:
                busy(streams[rng.integers(0, 3)], 4_000_000)
            if rng.random() < 0.1:
                busy(moves[rng.integers(0, 4)], 4_000_000)
            what = rng.choice(["admit", "fork", "fork", "resize", "resize", "resize", "compact", "suspend", "resume", "drop"])
            if what == "admit" and rid not in state:
                n = int(rng.integers(1, 70))
                if p.admit(rid, n)[0] == kvr.OK:
                    want[rid], owner[rid], state[rid] = np.zeros(n, np.uint8), s, kvr.ACTIVE
                    on_tokens(rid, 0, n)
            elif what == "fork" and rid not in state and state.get(other) == kvr.ACTIVE:
                n = int(rng.integers(0, len(want[other]) + 1))
                s.wait_stream(owner[other])                                       # the donor's tokens, as its owner wrote them
                if p.fork(rid, other, n, stream=s.cuda_stream)[0] == kvr.OK:
                    want[rid], owner[rid], state[rid] = want[other][:n].copy(), s, kvr.ACTIVE
                    done["fork"] += 1
            elif what == "resize" and state.get(rid) == kvr.ACTIVE:
                was, n = len(want[rid]), int(rng.integers(0, 90))
                if p.resize(rid, n, stream=owner[rid].cuda_stream)[0] == kvr.OK:
                    want[rid] = np.concatenate([want[rid][:n], np.zeros(max(0, n - was), np.uint8)])
                    if n > was:
                        on_tokens(rid, was, n)
                    done["resize"] += 1
            elif what == "compact":
                for t in streams:
                    s.wait_stream(t)
                done["compact"] += len(p.compact(int(rng.integers(0, 6)), stream=s.cuda_stream)[1])
                for t in streams:
                    t.wait_stream(s)
            elif what == "suspend" and state.get(rid) == kvr.ACTIVE:
                moves[1 if route == "dma2d" else 0].wait_stream(owner[rid])
                if p.suspend_to_host([rid])[0] == kvr.OK:
                    state[rid] = kvr.HOST
            elif what == "resume" and state.get(rid) == kvr.HOST:
                if p.resume_from_host([rid])[0] == kvr.OK:
                    state[rid] = kvr.ACTIVE
                    owner[rid].wait_stream(moves[2 if route == "dma2d" else 3])   # the owner's writes come behind the tokens that come back
                    done["resume"] += 1
            elif what == "drop" and rid in state:
                if state[rid] == kvr.ACTIVE:                                      # its stream may still write: the blocks go from there
                    assert p.resize(rid, 0, stream=owner[rid].cuda_stream)[0] == kvr.OK
                assert p.release(rid) == kvr.OK
                del want[rid], owner[rid], state[rid]
            if turn % 25 == 24:
                check()
        check()
    assert all(done.values()), done
