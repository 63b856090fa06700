"""One layer of a serving loop over a kvr pool: prefill, a step of drafted tokens, the wait for a human, and on.

    python examples/drafted_decode.py [bf16 | f16 | e4m3 | int8]

The pool's block tables and the cache operators work on the same memory: kvr.Pool hands out blocks and moves them to the
host and back, kvr.Cache writes tokens into them and attends over them.  Random numbers stand in for the projections.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2608_30830_b200 import kvr

Q_HEADS, KV_HEADS, DIM, BLOCK, BLOCKS, ROOM = 32, 8, 128, 16, 512, 64
# a tree of drafted tokens: each one's parent (the first follows the last accepted token)
PARENT = [-1, 0, 0, 1, 1, 2, 3, 3, 6]
ACCEPTED = [0, 2, 5]                       # the path that verification would keep


def ancestors():
    """Bit j of row i: drafted token i looks at drafted token j (its ancestors and itself)."""
    rows = []
    for i, p in enumerate(PARENT):
        rows.append((1 << i) | (rows[p] if p >= 0 else 0))
    return rows


def main(fmt="bf16"):
    device, dtype = "cuda", torch.float16 if fmt == "f16" else torch.bfloat16
    gen = torch.Generator(device).manual_seed(5)
    cache = kvr.Cache(1, KV_HEADS, DIM, BLOCK, BLOCKS, fmt)
    memory = torch.zeros(cache.pool_bytes, dtype=torch.uint8, device=device)
    workspace = torch.zeros(cache.workspace_bytes(), dtype=torch.uint8, device=device)   # zeroed once, used by every step
    table = torch.empty(4096, DIM // 2, 2, device=device)
    kvr.rope_table(table, base=500000.0)
    rope = kvr.Rope(table, DIM)
    status = torch.zeros(1, dtype=torch.int32, device=device)
    prompts = [700, 33, 1, 1290]

    with kvr.Pool(*cache.geometry, BLOCKS, 64 << 20, device_pool=memory.data_ptr()) as pool:
        for rid, n in enumerate(prompts):
            assert pool.admit(rid, n + ROOM)[0] == kvr.OK                # blocks for the prompt and what follows

        def batch(context, new):
            """The step's kvr_batch: `new[r]` tokens behind `context[r]`, under the pool's present block tables."""
            blocks = [pool.info(rid)[1]["blocks"] for rid in range(len(prompts))]
            width = max(len(b) for b in blocks)
            i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
            start = [0]
            for n in new:
                start.append(start[-1] + n)
            return kvr.Batch(i32(start), i32(context), i32([list(b) + [-1] * (width - len(b)) for b in blocks]), max(new),
                             max(c + n for c, n in zip(context, new)), status)

        def step(b, tokens, mask=None):
            """Projections (random here), append, attend."""
            qkv = torch.randn(tokens, Q_HEADS + 2 * KV_HEADS, DIM, generator=gen, device=device).to(dtype)
            q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], dim=1)    # views: strides are the operators' business
            turned, out = torch.empty(tokens, Q_HEADS, DIM, dtype=dtype, device=device), torch.empty(tokens, Q_HEADS, DIM, dtype=dtype, device=device)
            cache.append(memory, 0, b, q=q, k=k, v=v, q_out=turned, rope=rope)
            cache.attend(memory, 0, b, turned, out, workspace, mask=mask)
            return turned, out

        # prefill
        step(batch([0] * len(prompts), prompts), sum(prompts))
        # a step of drafted tokens: all of them appended, each attends to the context and its own branch
        rows = ancestors()
        mask = torch.tensor(rows * len(prompts), dtype=torch.int64, device=device)[:, None]
        drafted = batch(prompts, [len(PARENT)] * len(prompts))
        step(drafted, len(rows) * len(prompts), mask)
        # the accepted branch stays, packed behind the context; nothing else of the tree does
        index = torch.tensor([ACCEPTED] * len(prompts), dtype=torch.int32, device=device)
        cache.keep(memory, drafted, index, torch.full((len(prompts),), len(ACCEPTED), dtype=torch.int32, device=device))
        context = [n + len(ACCEPTED) for n in prompts]
        # one more token, once before and once after the requests have waited in host memory
        one = batch(context, [1] * len(prompts))
        turned, before = step(one, len(prompts))
        torch.cuda.synchronize()
        ids = list(range(len(prompts)))
        assert pool.suspend_to_host(ids, kvr.SYNC)[0] == kvr.OK
        memory.zero_()                     # what was there is the host's now
        torch.cuda.synchronize()
        assert pool.resume_from_host(ids, kvr.SYNC)[0] == kvr.OK
        after = torch.empty_like(before)
        cache.attend(memory, 0, batch(context, [1] * len(prompts)), turned, after, workspace)
        assert torch.equal(before, after), "the cache came back changed"
        # the way back to dense rows
        k, v = torch.empty(2, sum(context), KV_HEADS, DIM, dtype=dtype, device=device).unbind(0)
        cache.read(memory, 0, batch([0] * len(prompts), context), k, v)
        assert torch.isfinite(k).all() and torch.isfinite(v).all()
        assert status.item() == 0, "a device-side check failed"
    print("drafted decode ok (%s): %d requests, %d drafted tokens each, %d kept, suspended and resumed" %
          (fmt, len(prompts), len(PARENT), len(ACCEPTED)))
    return after


if __name__ == "__main__":
    main(*sys.argv[1:2])
