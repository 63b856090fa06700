"""Several answers to one prompt with a picture in it, over a kvr pool: prefill, fork, a token for each branch, and a pool without holes.

    python examples/forked_decode.py [e2m1 | bf16 | f16 | e4m3 | int8]

The branches share the prompt's full blocks; each has a last block of its own to write into.  The picture's tokens have positions of
three axes (time, height, width), the text's run together.  Random numbers stand in for the projections.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2608_30830_b200 import kvr

Q_HEADS, KV_HEADS, DIM, BLOCK, BLOCKS = 32, 8, 128, 16, 256
TEXT, PICTURE, BRANCHES = 61, (1, 18, 24), 4           # tokens of text before and behind a picture of 18 x 24 patches
AXES = [0] * 16 + [1] * 24 + [2] * 24                  # the axis of each pair of channels


def prompt_positions():
    """[tokens, 3] and the position that the answer goes on from."""
    text = torch.arange(TEXT)[:, None].expand(-1, 3)
    grid = torch.stack(torch.meshgrid(*[torch.arange(n) for n in PICTURE], indexing="ij"), -1).reshape(-1, 3) + TEXT
    behind = TEXT + max(PICTURE)
    return torch.cat([text, grid, text + behind]).int(), behind + TEXT


def main(fmt="e2m1"):
    device, dtype = "cuda", torch.float16 if fmt == "f16" else torch.bfloat16
    gen = torch.Generator(device).manual_seed(7)
    cache = kvr.Cache(1, KV_HEADS, DIM, BLOCK, BLOCKS, fmt)
    memory = torch.zeros(cache.pool_bytes, dtype=torch.uint8, device=device)
    workspace = torch.zeros(cache.workspace_bytes(), dtype=torch.uint8, device=device)
    table = torch.empty(4096, DIM // 2, 2, device=device)
    kvr.rope_table(table, base=500000.0)
    rope = kvr.Rope(table, DIM, axes=AXES)
    status = torch.zeros(1, dtype=torch.int32, device=device)
    where, behind = prompt_positions()
    n = len(where)
    stream = torch.cuda.current_stream().cuda_stream

    with kvr.Pool(*cache.geometry, BLOCKS, 64 << 20, device_pool=memory.data_ptr()) as pool:
        assert pool.admit(100, 300)[0] == kvr.OK                        # something that leaves a hole later
        assert pool.admit(0, n)[0] == kvr.OK

        def batch(ids, context, new):
            blocks = [pool.info(rid)[1]["blocks"] for rid in ids]
            width = max(len(b) for b in blocks)
            i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
            return kvr.Batch(i32([new * i for i in range(len(ids) + 1)]), i32([context] * len(ids)), i32([list(b) + [-1] * (width - len(b)) for b in blocks]),
                             new, context + new, status)

        def step(b, qkv, positions):
            q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], dim=1)
            turned, out = (torch.empty(len(qkv), Q_HEADS, DIM, dtype=dtype, device=device) for _ in range(2))
            cache.append(memory, 0, b, q=q, k=k, v=v, q_out=turned, rope=rope, positions=positions)
            cache.attend(memory, 0, b, turned, out, workspace)
            return turned, out

        random = lambda tokens: torch.randn(tokens, Q_HEADS + 2 * KV_HEADS, DIM, generator=gen, device=device).to(dtype)
        step(batch([0], 0, n), random(n), where.to(device))
        # the branches: the prompt's full blocks are shared, its last one is copied
        ids = list(range(BRANCHES))
        for rid in ids[1:]:
            assert pool.fork(rid, 0, n, stream=stream)[0] == kvr.OK
        assert pool.refcount(int(pool.info(0)[1]["blocks"][0])) == BRANCHES
        # a token for each, drawn differently
        for rid in ids:
            assert pool.resize(rid, n + 1, stream=stream)[0] == kvr.OK
        at = torch.full((BRANCHES, 3), behind, dtype=torch.int32, device=device)
        turned, before = step(batch(ids, n, 1), random(BRANCHES), at)
        # the hole closes; the answers stay what they are
        torch.cuda.synchronize()
        assert pool.release(100) == kvr.OK
        moved = pool.compact(stream=stream)[1]
        after = torch.empty_like(before)
        cache.attend(memory, 0, batch(ids, n, 1), turned, after, workspace)
        assert len(moved) > 0 and torch.equal(before, after), "the cache came back changed"
        # a branch takes its token back and waits on the host
        assert pool.resize(1, n, stream=stream)[0] == kvr.OK
        assert pool.suspend_to_host([1], kvr.SYNC)[0] == kvr.OK and pool.resume_from_host([1], kvr.SYNC)[0] == kvr.OK
        assert status.item() == 0, "a device-side check failed"
    print("forked decode ok (%s): a prompt of %d tokens, %d branches, %d blocks moved" % (fmt, n, BRANCHES, len(moved)))
    return after


if __name__ == "__main__":
    main(*sys.argv[1:2])
