"""Further operators over the paged cache as they are measured: a cache held in 4 bits (tokens written and read back, attention over
it), rotary positions with several axes, and copies of blocks.  Cases, plain forms in torch, and the calls a user makes.

A batch is a number of requests, each with a context already in the cache and some new tokens.  Pool layout:
bytes [layers][2][num_blocks][block_size][row].  A row of a 16-bit cache is [kv_heads][head_dim]; a row of a 4-bit one is
[kv_heads] records: head_dim / 2 bytes of e2m1 codes (channel 2i in the low half of byte i), one fp32 scale, one e4m3 scale for
each 16 channels, zeros up to a multiple of 16.  An element is code times its group's scale times the head's.
"""
import functools
import math
import statistics

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROPE_POSITIONS = 1 << 17
ROPE_BASE = 500000.0
CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LARGEST = 6.0 * 448.0                       # of a code times a group's scale
SMALLEST_SCALE = 2.0 ** -100
GROUP = 16


# ---- cases -------------------------------------------------------------------------

def _case(name, op, **kw):
    c = dict(name=name, op=op, fmt="e2m1", dtype="bf16", layers=1, q_heads=32, kv_heads=8, head_dim=128, block_size=16,
             n_req=1, context=1024, spread=0.0, new=1, new_spread=0.0, tree=False, rot=128, style="half", sections="", pairs=0, partial=False)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of 32 running requests, one token each: written, and handed on as the cache holds it; launch latency counts
        _case("4-bit write and read, a decode step", "append", n_req=32, context=2000, spread=0.6),
        # tensor-parallel rank with 2 KV heads, drafted tokens, half of the head turned
        _case("4-bit write and read, drafted", "append", dtype="f16", q_heads=16, kv_heads=2, n_req=32, context=2000, spread=0.6,
              new=13, rot=64, style="interleaved"),
        # a prefill step: ragged prompts, 28k tokens in all, whose dense attention takes K and V as the cache holds them
        _case("4-bit write and read, prefill", "append", n_req=7, context=0, new=4096, new_spread=0.5),
        # a decode step of requests that hold pictures: time, height, width
        _case("axes, a decode step", "axes", fmt="bf16", n_req=32, context=2000, spread=0.6, sections="16,24,24"),
        # prompts with pictures and video among the text, 16k tokens
        _case("axes, prefill", "axes", fmt="bf16", n_req=4, context=0, new=4096, new_spread=0.3, sections="16,24,24"),
        # the smallest answer: one request with a short context, one token
        _case("attend 4-bit, one short request", "attend", context=333),
        # decode of 32 requests with lognormal contexts (median 8192)
        _case("attend 4-bit, decode", "attend", n_req=32, context=8192, spread=0.6),
        # 8 x 128k tokens, blocks of 8
        _case("attend 4-bit, long", "attend", n_req=8, context=131072 - 1, block_size=8),
        # trees of 64 drafted tokens: 256 rows a KV head
        _case("attend 4-bit, tree of 64", "attend", n_req=16, context=8192, spread=0.3, new=64, tree=True),
        # requests that are forked at a block that is not full: the last block of each, its valid rows alone, all 32 layers
        _case("copy, forks", "copy", fmt="bf16", layers=32, n_req=8, pairs=8, partial=True),
        # a tensor-parallel rank's pool made compact: 3,000 blocks, e4m3, all 32 layers
        _case("copy, compaction", "copy", fmt="e4m3", layers=32, kv_heads=2, pairs=3000),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["append", "append", "axes", "axes", "attend", "attend", "attend", "attend", "copy"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    c = dict(op=op, fmt="e2m1", dtype=rng.choice(["bf16", "bf16", "f16"]), layers=1, kv_heads=kv_heads, q_heads=kv_heads * rng.choice([1, 2, 4, 4, 7, 8]),
             head_dim=rng.choice([64, 96, 128, 128, 128]), block_size=rng.choice([8, 16, 16, 32]), n_req=log_int(1, 64), spread=rng.choice([0.0, 0.3, 0.6]),
             new_spread=0.0, tree=False, style=rng.choice(["half", "interleaved"]), sections="", pairs=0, partial=False, new=1, context=0)
    c["rot"] = c["head_dim"] // rng.choice([1, 1, 2])
    if op in ("append", "axes"):
        new = log_int(1, 8192)
        c.update(new=new, new_spread=rng.choice([0.0, 0.5]) if new > 1 else 0.0, context=log_int(1, 2000))
        c["n_req"] = max(1, min(c["n_req"], 24_000 // new if op == "append" else 16_000 // new))
        if op == "axes":
            c["dtype"] = c["fmt"] = rng.choice(["bf16", "f16"])
            c["head_dim"] = rng.choice([64, 80, 128, 128])
            c["rot"] = c["head_dim"]
            pairs = c["rot"] // 2
            a, b = sorted(rng.sample(range(1, pairs), 2))
            c["sections"] = rng.choice(["16,24,24" if pairs == 64 else "%d,%d" % (pairs // 2, pairs - pairs // 2), "%d,%d,%d" % (a, b - a, pairs - b), "turns"])
    elif op == "attend":
        c["new"] = rng.choice([1, 1, 1, log_int(2, 64), log_int(2, 64)])
        c["tree"] = c["new"] > 1 and rng.random() < 0.8
        c["context"] = log_int(1, 131072)
        room = min(600_000, 100_000 * 64 * 32 // (c["new"] * c["q_heads"]))          # tokens of all requests
        c["context"] = min(c["context"], max(1, room // 2))
        c["n_req"] = max(1, min(c["n_req"], room // (c["context"] + c["new"])))
    else:
        c.update(fmt=rng.choice(["bf16", "e4m3", "e2m1"]), layers=rng.choice([8, 32, 64]), partial=rng.random() < 0.5)
        c["pairs"] = log_int(1, max(1, min(4000, 1_500_000_000 // (2 * c["layers"] * c["block_size"] * _row_bytes(c)))))
    return c


def _spread(n, median, sigma):
    """n lengths around a median: the quantiles of a lognormal distribution, clipped to a factor of four."""
    if median == 0:
        return [0] * n
    nd = statistics.NormalDist()
    return [max(1, min(4 * median, int(round(median * math.exp(sigma * nd.inv_cdf((i + 0.5) / n)))))) for i in range(n)]


def _lengths(case):
    """(context, new tokens) of each request; the order is fixed, long and short ones mixed."""
    n = case["n_req"]
    order = sorted(range(n), key=lambda i: (i * 37 + 11) % 101)
    context, new = _spread(n, case["context"], case["spread"]), _spread(n, case["new"], case["new_spread"])
    return [context[i] for i in order], [new[n - 1 - i] for i in order]


def _record_bytes(case):
    """A head's record in a 4-bit row."""
    d = case["head_dim"]
    return -(-(d // 2 + 4 + d // GROUP) // 16) * 16


def _row_bytes(case):
    h, d = case["kv_heads"], case["head_dim"]
    if case["fmt"] == "e2m1":
        return h * _record_bytes(case)
    return h * d * 2 if case["fmt"] in ("bf16", "f16") else h * d + -(-4 * h // 16) * 16


def _rows_copied(case):
    """Rows of each pair's block that are copied."""
    bs = case["block_size"]
    return [1 + (i * 5 + 2) % bs if case["partial"] else bs for i in range(case["pairs"])]


def _axes(case):
    """The axis of each rotated pair, from its sections; "turns" deals three axes out in turn."""
    pairs = case["rot"] // 2
    if case["sections"] == "turns":
        return [p % 3 for p in range(pairs)]
    return [axis for axis, n in enumerate(case["sections"].split(",")) for _ in range(int(n))]


def work(case):
    h, hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    if case["op"] == "copy":
        return {"bytes": 2 * 2 * case["layers"] * sum(_rows_copied(case)) * _row_bytes(case), "flops": 0}
    context, new = _lengths(case)
    tokens, row = sum(new), h * (d // 2 + 4 + d // GROUP) if case["fmt"] == "e2m1" else h * d * 2   # without the padding
    if case["op"] == "attend":
        pairs = sum((c + t) * t for c, t in zip(context, new)) * hq
        return {"bytes": sum(c + t for c, t in zip(context, new)) * 2 * row + tokens * hq * (2 * d * 2 + 4), "flops": 4 * d * pairs}
    read_back = 2 * h * d * 2 + 2 * row if case["op"] == "append" else 0
    return {"bytes": tokens * (2 * hq * d * 2 + 2 * h * d * 2 + 2 * row + case["rot"] * 4 + read_back), "flops": tokens * 3 * (hq + h) * case["rot"]}


# ---- the pool's layout -------------------------------------------------------------

def _rows(pool, case):
    """The pool as [layers * 2][slots][row bytes]."""
    return pool.view(2 * case["layers"], -1, _row_bytes(case))


def _elements(pool, case):
    """A 16-bit pool's elements, [planes][slots][kv_heads][head_dim], as a view."""
    return _rows(pool, case).view(TYPES[case["fmt"]]).unflatten(-1, (case["kv_heads"], case["head_dim"]))


def _records(pool, case):
    """A 4-bit pool's records, [planes][slots][kv_heads][record bytes]."""
    return _rows(pool, case).unflatten(-1, (case["kv_heads"], _record_bytes(case)))


def _scales(pool, case):
    """The heads' scales of a 4-bit pool, [planes][slots][kv_heads], as a view."""
    d = case["head_dim"]
    return _records(pool, case)[..., d // 2:d // 2 + 4].view(torch.float32)[..., 0]


def _groups(pool, case):
    """The groups' scales of a 4-bit pool, [planes][slots][kv_heads][groups], as a view."""
    d = case["head_dim"]
    return _records(pool, case)[..., d // 2 + 4:d // 2 + 4 + d // GROUP].view(torch.float8_e4m3fn)


def _pack(x):
    """Records of x [..., head_dim] in fp32: (codes in pairs as bytes, groups' scales, heads' scales)."""
    g = x.unflatten(-1, (-1, GROUP))
    scale = torch.clamp(x.abs().amax(-1, keepdim=True) * torch.tensor(1.0 / LARGEST, dtype=torch.float32, device=x.device), min=SMALLEST_SCALE)
    sixth = torch.tensor(1.0 / 6.0, dtype=torch.float32, device=x.device)
    group = torch.clamp(g.abs().amax(-1) * (1.0 / scale * sixth), max=448.0).to(torch.float8_e4m3fn)
    step = group.float() * scale
    y = g * torch.where(step > 0, 1.0 / step, torch.zeros_like(step))[..., None]
    a = y.abs()
    # to the nearest code, ties to the even one: steps of a half up to 2, of one up to 4, of two up to 6
    code = torch.where(a <= 2, (a * 2).round(), torch.where(a <= 4, a.round() + 2, torch.clamp((a / 2).round() + 4, max=7))).to(torch.uint8)
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), group, scale[..., 0]


@functools.lru_cache(maxsize=None)
def _code_values():
    return torch.tensor(CODES + tuple(-c for c in CODES), dtype=torch.float32, device=DEVICE)


def _unpack(records, d, kind=torch.float32):
    """The values [..., head_dim] that records stand for."""
    byte = records[..., :d // 2]
    codes = torch.stack([byte & 15, byte >> 4], -1).flatten(-2)
    group = records[..., d // 2 + 4:d // 2 + 4 + d // GROUP].contiguous().view(torch.float8_e4m3fn).to(kind)
    scale = records[..., d // 2:d // 2 + 4].contiguous().view(torch.float32).to(kind)
    return (_code_values().to(kind)[codes.int()].unflatten(-1, (-1, GROUP)) * group[..., None]).flatten(-2) * scale


# ---- inputs ------------------------------------------------------------------------

def _fill(pool, case, gen):
    """A cache as a model leaves it: channels of unlike size in K, tokens of unlike size in V."""
    h, d = case["kv_heads"], case["head_dim"]
    slots = _rows(pool, case).shape[1]
    for plane in range(2 * case["layers"]):
        for at in range(0, slots, 1 << 18):
            n = min(1 << 18, slots - at)
            x = torch.randn((n, h, d), device=DEVICE, generator=gen)
            channels = torch.Generator(device=DEVICE).manual_seed(plane)
            x *= torch.exp(0.4 * torch.randn((h, d) if plane % 2 == 0 else (n, 1, 1), device=DEVICE, generator=channels if plane % 2 == 0 else gen))
            if case["fmt"] == "e2m1":
                codes, group, scale = _pack(x)
                _records(pool, case)[plane, at:at + n, :, :d // 2] = codes
                _groups(pool, case)[plane, at:at + n] = group
                _scales(pool, case)[plane, at:at + n] = scale
            else:
                _elements(pool, case)[plane, at:at + n] = x.to(TYPES[case["fmt"]])


@functools.lru_cache(maxsize=8)
def _rope_table(rot):
    """cos and sin of every position, [positions][rot / 2][2] in fp32, from angles in fp64."""
    freq = ROPE_BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / rot)
    angle = torch.arange(ROPE_POSITIONS, dtype=torch.float64, device=DEVICE)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def _parents(n, rng):
    """A tree of n drafted tokens: the parent of each (-1 for the root), a chain with side branches."""
    return [-1] + [i - 1 if rng.random() < 0.5 else int(rng.integers(0, i)) for i in range(1, n)]


def _places(length, axes, rng):
    """Positions of a request's tokens, [length][axes]: text, where all axes run together, and pictures, whose tokens lie on a grid that
    the text behind them goes on from."""
    at, start, parts = 0, 0, []
    while at < length:
        n = min(length - at, int(rng.integers(1, 400)))
        parts.append(np.repeat(np.arange(start, start + n)[:, None], axes, 1))
        at, start = at + n, start + n
        if at < length:
            frames, rows, columns = int(rng.integers(1, 5)), int(rng.integers(4, 33)), int(rng.integers(4, 33))
            grid = np.indices((frames, rows, columns)).reshape(3, -1).T[:, 3 - axes:]
            parts.append(start + grid[:length - at])
            at, start = at + len(parts[-1]), start + max(frames, rows, columns)
    return np.concatenate(parts).astype(np.int32)


def _prepare_copy(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    num_blocks = 2 * case["pairs"] + case["pairs"] // 4 + 1
    ids = rng.permutation(num_blocks)[:2 * case["pairs"]].astype(np.int32).reshape(case["pairs"], 2)
    size = 2 * case["layers"] * num_blocks * case["block_size"] * _row_bytes(case)
    st = dict(case=case, num_blocks=num_blocks, pairs=torch.from_numpy(ids).to(DEVICE), rows=None)
    st["pool"] = torch.randint(0, 256, (size,), dtype=torch.uint8, device=DEVICE, generator=gen)
    if case["partial"]:
        st["rows"] = torch.tensor(_rows_copied(case), dtype=torch.int32, device=DEVICE)
    return st


def prepare(case, seed):
    if case["op"] == "copy":
        return _prepare_copy(case, seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    context, new = _lengths(case)
    n, bs = case["n_req"], case["block_size"]
    blocks = [-(-(c + t) // bs) for c, t in zip(context, new)]
    num_blocks = sum(blocks) + sum(blocks) // 4 + 1
    ids = rng.permutation(num_blocks)[:sum(blocks)].astype(np.int32)
    tables = np.zeros((n, max(blocks)), dtype=np.int32)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    at = 0
    for r, k in enumerate(blocks):
        tables[r, :k] = ids[at:at + k]
        at += k
    st = dict(case=case, num_blocks=num_blocks, max_new=max(new), max_tokens=max(c + t for c, t in zip(context, new)),
              tables=torch.from_numpy(tables).to(DEVICE), token_start=torch.from_numpy(starts).to(DEVICE),
              context=torch.tensor(context, dtype=torch.int32, device=DEVICE))
    # where each new token lies: its request, and its place among the request's tokens
    req = np.repeat(np.arange(n), new)
    place = np.concatenate([np.arange(c, c + t) for c, t in zip(context, new)])
    st["slots"] = torch.from_numpy(tables[req, place // bs].astype(np.int64) * bs + place % bs).to(DEVICE)
    st["pool"] = torch.zeros(2 * case["layers"] * num_blocks * bs * _row_bytes(case), dtype=torch.uint8, device=DEVICE)
    _fill(st["pool"], case, gen)
    tokens, h, hq, d = int(starts[-1]), case["kv_heads"], case["q_heads"], case["head_dim"]
    kind = TYPES[case["dtype"]]
    if case["op"] in ("append", "axes"):
        # as a projection leaves them: q, k and v are parts of one tensor
        qkv = torch.randn(tokens, hq + 2 * h, d, device=DEVICE, generator=gen)
        qkv[:, hq:hq + h] *= torch.exp(0.4 * torch.randn(h, d, device=DEVICE, generator=gen))
        qkv = qkv.to(kind)
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + h], v=qkv[:, hq + h:], q_out=torch.zeros(tokens, hq, d, dtype=kind, device=DEVICE),
                  rope=_rope_table(case["rot"]))
        if case["op"] == "append":
            st.update(positions=torch.from_numpy(place.astype(np.int32)).to(DEVICE), k_out=torch.zeros(tokens, h, d, dtype=kind, device=DEVICE),
                      v_out=torch.zeros(tokens, h, d, dtype=kind, device=DEVICE))
        else:
            axes = max(_axes(case)) + 1
            where = np.concatenate([_places(c + t, axes, rng)[c:] for c, t in zip(context, new)])
            st.update(positions=torch.from_numpy(where).to(DEVICE), axes=_axes(case))
    else:
        st.update(q=(1.2 * torch.randn(tokens, hq, d, device=DEVICE, generator=gen)).to(kind), scale=1.0 / math.sqrt(d),
                  out=torch.zeros(tokens, hq, d, dtype=kind, device=DEVICE), lse=torch.zeros(tokens, hq, device=DEVICE), mask=None)
        if case["tree"]:
            words = -(-max(new) // 64)
            mask = np.zeros((tokens, words * 64), dtype=bool)
            for r, t in enumerate(new):
                rows = mask[starts[r]:starts[r] + t]
                for i, p in enumerate(_parents(t, rng)):
                    if p >= 0:
                        rows[i] = rows[p]
                    rows[i, i] = True
            st["mask"] = torch.from_numpy(np.packbits(mask, axis=1, bitorder="little").view(np.int64)).to(DEVICE)
    return st


# ---- the framework's operators -----------------------------------------------------

@functools.lru_cache(maxsize=None)
def _cache(layers, kv_heads, head_dim, block_size, num_blocks, fmt):
    """The description of a cache, made once as a program does; it holds no data."""
    from paper_2608_30830_b200 import kvr
    return kvr.Cache(layers, kv_heads, head_dim, block_size, num_blocks, fmt)


@functools.lru_cache(maxsize=None)
def _workspace(cache):
    """Attention's workspace, one for a cache."""
    return torch.zeros(cache.workspace_bytes(), dtype=torch.uint8, device=DEVICE)


def _run_own(st):
    from paper_2608_30830_b200 import kvr
    case = st["case"]
    cache = _cache(case["layers"], case["kv_heads"], case["head_dim"], case["block_size"], st["num_blocks"], case["fmt"])
    if case["op"] == "copy":
        cache.copy(st["pool"], st["pairs"], rows=st["rows"])
        return
    batch = kvr.Batch(st["token_start"], st["context"], st["tables"], st["max_new"], st["max_tokens"])
    if case["op"] == "append":
        rope = kvr.Rope(st["rope"], case["rot"], case["style"])
        cache.append(st["pool"], 0, batch, q=st["q"], k=st["k"], v=st["v"], q_out=st["q_out"], rope=rope, positions=st["positions"])
        cache.read(st["pool"], 0, batch, st["k_out"], st["v_out"])
    elif case["op"] == "axes":
        rope = kvr.Rope(st["rope"], case["rot"], case["style"], axes=st["axes"])
        cache.append(st["pool"], 0, batch, q=st["q"], k=st["k"], v=st["v"], q_out=st["q_out"], rope=rope, positions=st["positions"])
    else:
        cache.attend(st["pool"], 0, batch, st["q"], st["out"], _workspace(cache), lse=st["lse"], mask=st["mask"], scale=st["scale"])


# ---- plain forms -------------------------------------------------------------------

def _rotate(x, st):
    """x [tokens, heads, head_dim] in fp32, its first `rot` channels turned by each token's position (of the pair's axis)."""
    case = st["case"]
    rot = case["rot"]
    if case["op"] == "axes":
        pair = torch.arange(rot // 2, device=DEVICE)
        angles = st["rope"][st["positions"].long()[:, torch.tensor(st["axes"], device=DEVICE)], pair]
    else:
        angles = st["rope"][st["positions"].long()]
    cos, sin = angles.unbind(-1)
    cos, sin = cos[:, None], sin[:, None]
    if case["style"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _put_records(st, plane, x):
    case = st["case"]
    d = case["head_dim"]
    codes, group, scale = _pack(x)
    records = _records(st["pool"], case)[plane]
    record = torch.zeros(x.shape[:2] + (_record_bytes(case),), dtype=torch.uint8, device=DEVICE)
    record[..., :d // 2] = codes
    record[..., d // 2:d // 2 + 4] = scale[..., None].contiguous().view(torch.uint8)
    record[..., d // 2 + 4:d // 2 + 4 + d // GROUP] = group.view(torch.uint8)
    records[st["slots"]] = record


def _append_plain(st):
    case = st["case"]
    st["q_out"].copy_(_rotate(st["q"].float(), st))
    turned, v = _rotate(st["k"].float(), st), st["v"].float()
    if case["op"] == "axes":
        cache = _elements(st["pool"], case)
        cache[0][st["slots"]] = turned.to(cache.dtype)
        cache[1][st["slots"]] = v.to(cache.dtype)
        return
    _put_records(st, 0, turned)
    _put_records(st, 1, v)
    st["k_out"].copy_(_unpack(_records(st["pool"], case)[0][st["slots"]], case["head_dim"]))
    st["v_out"].copy_(_unpack(_records(st["pool"], case)[1][st["slots"]], case["head_dim"]))


def _attend_plain(st):
    case = st["case"]
    n, bs, h, hq, d = case["n_req"], case["block_size"], case["kv_heads"], case["q_heads"], case["head_dim"]
    g, t, m = hq // h, st["max_new"], st["max_tokens"]
    start, context = st["token_start"].long(), st["context"].long()
    count = start[1:] - start[:-1]
    key = torch.arange(m, device=DEVICE)
    slots = st["tables"].long()[:, key // bs] * bs + key % bs                              # [n, m]
    row = torch.arange(t, device=DEVICE)
    token = torch.clamp(start[:-1, None] + row, max=int(st["q"].shape[0]) - 1)            # [n, t]
    rel = key - context[:, None]                                                           # [n, m]: < 0 is context
    if st["mask"] is None:
        new = rel[:, None] <= row[:, None]
    else:
        at = torch.clamp(rel, 0, t - 1)
        word = st["mask"][token][:, :, None].expand(-1, -1, m, -1).gather(3, (at // 64)[:, None, :, None].expand(-1, t, -1, 1))[..., 0]
        new = (word >> (at % 64)[:, None]) & 1 == 1
    seen = ((rel < 0)[:, None] | new) & (rel < count[:, None])[:, None]                     # [n, t, m]
    records = _records(st["pool"], case)
    q = st["q"][token].float().unflatten(2, (h, g)).permute(0, 2, 3, 1, 4).reshape(n, h, g * t, d)
    s = torch.matmul(q, _unpack(records[0][slots], d).permute(0, 2, 3, 1)).view(n, h, g, t, m)
    s = (s * st["scale"]).masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, h, g * t, m), _unpack(records[1][slots], d).transpose(1, 2)).view(n, h, g, t, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    real = row < count[:, None]                                                             # [n, t]
    st["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(n, t, hq, d)[real])
    st["lse"].copy_((top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(n, t, hq)[real])


def _copy_plain(st):
    case = st["case"]
    rows = _rows(st["pool"], case)
    row = torch.arange(case["block_size"], device=DEVICE)
    slots = st["pairs"].long()[:, :, None] * case["block_size"] + row                      # [pairs, 2, block_size]
    kept = (row < st["rows"][:, None]) if st["rows"] is not None else torch.ones_like(slots[:, 0], dtype=torch.bool)
    rows[:, slots[:, 1][kept]] = rows[:, slots[:, 0][kept]]


def _run_plain(st):
    op = st["case"]["op"]
    (_append_plain if op in ("append", "axes") else _attend_plain if op == "attend" else _copy_plain)(st)


def run(state):
    (_run_own if own else _run_plain)(state)
    case = state["case"]
    if case["op"] == "append":
        # what the cache holds of the new tokens by value; the scales of all
        return {"q": state["q_out"], "k": state["k_out"], "v": state["v_out"], "scales": _scales(state["pool"], case), "groups": _groups(state["pool"], case)}
    if case["op"] == "axes":
        return {"q": state["q_out"], "cache": _elements(state["pool"], case)}
    if case["op"] == "attend":
        return {"out": state["out"], "lse": state["lse"]}
    return {"pool": state["pool"].view(torch.int32)}


# ---- the definition in 64 bits -----------------------------------------------------

def exact(case, seed):
    if case["op"] == "copy":
        return None                                                     # bytes move as they are
    st = prepare(case, seed)
    op, d = case["op"], case["head_dim"]
    bs, h, hq = case["block_size"], case["kv_heads"], case["q_heads"]
    if op in ("append", "axes"):
        # a pair of channels as a complex number, times exp(i * angle)
        rot = case["rot"]
        freq = ROPE_BASE ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=DEVICE) / rot)
        where = st["positions"].double()
        angle = (where[:, st["axes"]] if op == "axes" else where[:, None]) * freq
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]

        def turned(x):
            x = x.double().clone()
            first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["style"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            x[..., first], x[..., second] = z.real, z.imag
            return x

        rows, out = [turned(st["k"]), st["v"].double()], {"q": turned(st["q"])}
        if op == "axes":
            out["cache"] = _elements(st["pool"], case).double()
            for plane, x in enumerate(rows):
                out["cache"][plane][st["slots"]] = x
        else:
            # codes and groups' scales are rounded values; q and the heads' scales have 64-bit ones
            scales = _scales(st["pool"], case).double()
            for plane, x in enumerate(rows):
                scales[plane][st["slots"]] = x.abs().amax(-1) / LARGEST
            out.update(k=None, v=None, groups=None, scales=scales)
        return out
    if sum(work(case).values()) > 2e12:
        return None
    out, lse = [], []
    context, new = _lengths(case)
    at = 0
    for r, (c, t) in enumerate(zip(context, new)):
        j = torch.arange(c + t, device=DEVICE)
        slots = st["tables"][r].long()[j // bs] * bs + j % bs
        kv = [_unpack(_records(st["pool"], case)[plane][slots], d, torch.float64).transpose(0, 1) for plane in (0, 1)]      # [h, c + t, d]
        seen = torch.ones(t, c + t, dtype=torch.bool, device=DEVICE)
        if st["mask"] is None:
            seen[:, c:] = torch.ones(t, t, dtype=torch.bool, device=DEVICE).tril()
        else:
            bits = np.unpackbits(st["mask"][at:at + t].cpu().numpy().view(np.uint8), axis=1, bitorder="little")
            seen[:, c:] = torch.from_numpy(bits[:, :t].astype(bool)).to(DEVICE)
        o_r = torch.empty(t, hq, d, dtype=torch.float64, device=DEVICE)
        l_r = torch.empty(t, hq, dtype=torch.float64, device=DEVICE)
        for head in range(hq):
            k, v = (x[head // (hq // h)] for x in kv)
            s = (st["q"][at:at + t, head].double() @ k.T * st["scale"]).masked_fill(~seen, -math.inf)
            l_r[:, head] = torch.logsumexp(s, -1)
            o_r[:, head] = torch.exp(s - l_r[:, head, None]) @ v
        out.append(o_r)
        lse.append(l_r)
        at += t
    return {"out": torch.cat(out), "lse": torch.cat(lse)}
