"""The operators over the paged cache as they are measured: cases, plain forms in torch, and the calls a user makes.

A batch is a number of requests, each with a context already in the cache and some new tokens.  Pool layout:
bytes [layers][2][num_blocks][block_size][row]; a row of a 16-bit cache is [kv_heads][head_dim], a row of a
quantised one is the codes of all heads followed by one fp32 scale a head, padded to 16 bytes.
"""
import functools
import math
import statistics

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FORMATS = {"bf16": (torch.bfloat16, 2), "f16": (torch.float16, 2), "e4m3": (torch.float8_e4m3fn, 1), "int8": (torch.int8, 1)}
LARGEST_CODE = {"e4m3": 448.0, "int8": 127.0}
ROPE_POSITIONS = 1 << 17
SMALLEST_SCALE = 2.0 ** -126


# ---- cases -------------------------------------------------------------------------

def _case(name, op, **kw):
    c = dict(name=name, op=op, fmt="bf16", dtype="bf16", layers=1, q_heads=32, kv_heads=8, head_dim=128, block_size=16,
             n_req=1, context=1024, spread=0.0, new=1, new_spread=0.0, tree=False, rot=128, style="half")
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of 32 running requests: one token each, 32 query / 8 KV heads; launch latency counts
        _case("append, a decode step", "append", n_req=32, context=2000, spread=0.6),
        # tensor-parallel rank with 2 KV heads writing drafted tokens into an int8 cache; interleaved, half the head
        _case("append, drafted, int8", "append", fmt="int8", q_heads=16, kv_heads=2, n_req=32, context=2000, spread=0.6,
              new=13, rot=64, style="interleaved"),
        # a prefill step: ragged prompts, 32k tokens in all, into an e4m3 cache
        _case("append, prefill, e4m3", "append", fmt="e4m3", n_req=7, context=0, new=4096, new_spread=0.5),
        # one 8,192-token request read back for a dense consumer
        _case("read, one request, e4m3", "read", fmt="e4m3", context=0, new=8192),
        # 32 ragged requests of an int8 cache, read back as fp16
        _case("read, batch, int8", "read", fmt="int8", dtype="f16", n_req=32, context=0, new=8192, new_spread=0.6),
        # the smallest answer: one request with a short context, one token
        _case("attend, one short request", "attend", context=333),
        # decode of 32 requests with lognormal contexts (median 8192): bound by reading the cache
        _case("attend, decode", "attend", n_req=32, context=8192, spread=0.6),
        # 8 x 128k tokens, blocks of 8, cache in e4m3
        _case("attend, long, e4m3", "attend", fmt="e4m3", n_req=8, context=131072 - 1, block_size=8),
        # tensor-parallel rank (2 KV heads, 16 query heads): trees of 13 drafted tokens over an int8 cache
        _case("attend, tree of 13, int8", "attend", fmt="int8", q_heads=16, kv_heads=2, n_req=32, context=8400, spread=0.3,
              new=13, tree=True),
        # trees of 64 drafted tokens: 256 rows a KV head, bound by the matrix units as much as by the cache
        _case("attend, tree of 64", "attend", n_req=16, context=8192, spread=0.3, new=64, tree=True),
        # accepted tokens of a few requests, all 32 layers
        _case("keep, few requests", "keep", layers=32, n_req=4, context=200, spread=0.3, new=8),
        # accepted tokens of 64 requests with trees of 64, e4m3 cache
        _case("keep, many requests, e4m3", "keep", fmt="e4m3", layers=32, n_req=64, context=200, spread=0.3, new=64),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["append", "append", "read", "attend", "attend", "attend", "attend", "keep"])
    fmt = rng.choice(["bf16", "bf16", "f16", "e4m3", "int8"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    c = dict(op=op, fmt=fmt, dtype=fmt if fmt in ("bf16", "f16") else rng.choice(["bf16", "f16"]), layers=1, kv_heads=kv_heads,
             q_heads=kv_heads * rng.choice([1, 2, 4, 4, 7, 8]), head_dim=rng.choice([64, 128, 128, 128]), block_size=rng.choice([8, 16, 16, 32]),
             n_req=log_int(1, 64), spread=rng.choice([0.0, 0.3, 0.6]), new_spread=0.0, tree=False, style=rng.choice(["half", "interleaved"]))
    c["rot"] = c["head_dim"] // rng.choice([1, 1, 2])
    if op in ("append", "read"):
        new = log_int(1, 8192)
        c.update(new=new, new_spread=rng.choice([0.0, 0.5]) if new > 1 else 0.0, context=log_int(1, 2000) if op == "append" else 0)
        c["n_req"] = max(1, min(c["n_req"], 150_000 // new))
    elif op == "attend":
        c["new"] = rng.choice([1, 1, 1, log_int(2, 64), log_int(2, 64)])
        c["tree"] = c["new"] > 1 and rng.random() < 0.8
        c["context"] = log_int(1, 131072)
        room = min(600_000, 100_000 * 64 * 32 // (c["new"] * c["q_heads"]))          # tokens of all requests
        c["context"] = min(c["context"], max(1, room // 2))
        c["n_req"] = max(1, min(c["n_req"], room // (c["context"] + c["new"])))
    else:
        c.update(layers=rng.choice([8, 32, 64]), context=log_int(1, 400), new=log_int(2, 64))
        c["n_req"] = max(1, min(c["n_req"], 600_000 // (c["layers"] * (c["context"] + c["new"]))))
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


def _kept(new, i):
    """How many of a request's drafted tokens are accepted: one to a third of them."""
    return 1 + (i * 7) % max(1, -(-new // 3))


def _row_bytes(case):
    h, d = case["kv_heads"], case["head_dim"]
    return h * d * 2 if FORMATS[case["fmt"]][1] == 2 else h * d + -(-4 * h // 16) * 16


def work(case):
    context, new = _lengths(case)
    row, h, hq, d = _row_bytes(case), case["kv_heads"], case["q_heads"], case["head_dim"]
    e = 4 if case["dtype"] == "f32" else 2
    tokens = sum(new)
    if case["fmt"] in LARGEST_CODE:
        row = h * d + 4 * h                                         # without the padding
    if case["op"] == "append":
        return {"bytes": tokens * (2 * hq * d * e + 2 * h * d * e + 2 * row + case["rot"] * 4), "flops": tokens * 3 * (hq + h) * case["rot"]}
    if case["op"] == "read":
        return {"bytes": tokens * 2 * (row + h * d * e), "flops": 0}
    if case["op"] == "attend":
        pairs = sum((c + t) * t for c, t in zip(context, new)) * hq
        return {"bytes": sum(c + t for c, t in zip(context, new)) * 2 * row + tokens * hq * (2 * d * e + 4), "flops": 4 * d * pairs}
    moved = sum(_kept(t, i) for i, t in enumerate(new))
    return {"bytes": moved * 2 * 2 * case["layers"] * row, "flops": 0}


# ---- inputs ------------------------------------------------------------------------

def _rows(pool, case):
    """The pool as [layers * 2][slots][row bytes]."""
    return pool.view(2 * case["layers"], -1, _row_bytes(case))


def _codes(pool, case):
    """The pool's elements, [planes][slots][kv_heads][head_dim], as a view of their own type."""
    h, d = case["kv_heads"], case["head_dim"]
    kind, size = FORMATS[case["fmt"]]
    return _rows(pool, case)[..., :h * d * size].view(kind).unflatten(-1, (h, d))


def _scales(pool, case):
    """The scales of a quantised pool, [planes][slots][kv_heads]."""
    h, d = case["kv_heads"], case["head_dim"]
    return _rows(pool, case)[..., h * d:h * d + 4 * h].view(torch.float32)


def _fill(pool, case, gen):
    """A cache as a model leaves it: channels of unlike size in K, tokens of unlike size in V."""
    h, d = case["kv_heads"], case["head_dim"]
    codes = _codes(pool, case)
    for plane in range(codes.shape[0]):
        x = torch.randn(codes.shape[1:], device=DEVICE, generator=gen)
        size = (h, d) if plane % 2 == 0 else (x.shape[0], 1, 1)
        x *= torch.exp(0.4 * torch.randn(size, device=DEVICE, generator=gen))
        if case["fmt"] in LARGEST_CODE:
            s = torch.clamp(x.abs().amax(-1, keepdim=True) / LARGEST_CODE[case["fmt"]], min=SMALLEST_SCALE)
            _scales(pool, case)[plane] = s[..., 0]
            x /= s
            x = x.round_() if case["fmt"] == "int8" else x
        codes[plane] = x.to(codes.dtype)


@functools.lru_cache(maxsize=8)
def _rope_table(rot):
    """cos and sin of every position, [positions][rot / 2][2] in fp32, from angles in fp64."""
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / rot)
    angle = torch.arange(ROPE_POSITIONS, dtype=torch.float64, device=DEVICE)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def _parents(n, rng):
    """A tree of n drafted tokens: the parent of each (-1 for the root), a chain with side branches."""
    return [-1] + [i - 1 if rng.random() < 0.5 else int(rng.integers(0, i)) for i in range(1, n)]


def prepare(case, seed):
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
    if case["op"] == "append":
        # as a projection leaves them: q, k and v are parts of one tensor
        qkv = torch.randn(tokens, hq + 2 * h, d, device=DEVICE, generator=gen)
        qkv[:, hq:hq + h] *= torch.exp(0.4 * torch.randn(h, d, device=DEVICE, generator=gen))
        qkv = qkv.to(kind)
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + h], v=qkv[:, hq + h:], q_out=torch.zeros(tokens, hq, d, dtype=kind, device=DEVICE),
                  positions=torch.from_numpy(place.astype(np.int32)).to(DEVICE), rope=_rope_table(case["rot"]))
    elif case["op"] == "read":
        st.update(k_out=torch.zeros(tokens, h, d, dtype=kind, device=DEVICE), v_out=torch.zeros(tokens, h, d, dtype=kind, device=DEVICE))
    elif case["op"] == "attend":
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
    else:
        count = [_kept(t, i) for i, t in enumerate(new)]
        index = np.zeros((n, max(count)), dtype=np.int32)
        for r, (t, k) in enumerate(zip(new, count)):
            index[r, :k] = np.sort(rng.permutation(t)[:k])
        st.update(index=torch.from_numpy(index).to(DEVICE), count=torch.tensor(count, dtype=torch.int32, device=DEVICE))
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
    batch = kvr.Batch(st["token_start"], st["context"], st["tables"], st["max_new"], st["max_tokens"])
    if case["op"] == "append":
        rope = kvr.Rope(st["rope"], case["rot"], case["style"])
        cache.append(st["pool"], 0, batch, q=st["q"], k=st["k"], v=st["v"], q_out=st["q_out"], rope=rope, positions=st["positions"])
    elif case["op"] == "read":
        cache.read(st["pool"], 0, batch, st["k_out"], st["v_out"])
    elif case["op"] == "attend":
        cache.attend(st["pool"], 0, batch, st["q"], st["out"], _workspace(cache), lse=st["lse"], mask=st["mask"], scale=st["scale"])
    else:
        cache.keep(st["pool"], batch, st["index"], st["count"])


# ---- plain forms -------------------------------------------------------------------

def _rotate(x, st):
    """x [tokens, heads, head_dim] in fp32, its first `rot` channels turned by each token's position."""
    case = st["case"]
    rot = case["rot"]
    cos, sin = st["rope"][st["positions"].long()].unbind(-1)
    cos, sin = cos[:, None], sin[:, None]
    if case["style"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _put(st, plane, x):
    case = st["case"]
    codes = _codes(st["pool"], case)[plane]
    if case["fmt"] in LARGEST_CODE:
        s = torch.clamp(x.abs().amax(-1, keepdim=True) / LARGEST_CODE[case["fmt"]], min=SMALLEST_SCALE)
        _scales(st["pool"], case)[plane][st["slots"]] = s[..., 0]
        x = x / s
        x = x.round() if case["fmt"] == "int8" else x
    # a byte view where the elements are bytes: indexed writes know no 8-bit floats
    x = x.to(codes.dtype)
    if codes.dtype == torch.float8_e4m3fn:
        codes, x = codes.view(torch.uint8), x.view(torch.uint8)
    codes[st["slots"]] = x


def _get(st, plane, slots):
    """The elements at `slots`, in fp32."""
    case = st["case"]
    codes = _codes(st["pool"], case)[plane]
    if codes.dtype == torch.float8_e4m3fn:
        x = codes.view(torch.uint8)[slots].view(torch.float8_e4m3fn).float()
    else:
        x = codes[slots].float()
    return x * _scales(st["pool"], case)[plane][slots][..., None] if case["fmt"] in LARGEST_CODE else x


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
    q = st["q"][token].float().unflatten(2, (h, g)).permute(0, 2, 3, 1, 4).reshape(n, h, g * t, d)
    s = torch.matmul(q, _get(st, 0, slots).permute(0, 2, 3, 1)).view(n, h, g, t, m)
    s = (s * st["scale"]).masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, h, g * t, m), _get(st, 1, slots).transpose(1, 2)).view(n, h, g, t, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    real = row < count[:, None]                                                             # [n, t]
    st["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(n, t, hq, d)[real])
    st["lse"].copy_((top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(n, t, hq)[real])


def _keep_plain(st):
    case = st["case"]
    bs = case["block_size"]
    i = torch.arange(st["index"].shape[1], device=DEVICE)
    context = st["context"].long()[:, None]
    source, target = context + st["index"].long(), (context + i).expand(case["n_req"], -1)
    tables = st["tables"].long()
    kept = i < st["count"][:, None]
    source = (tables.gather(1, torch.clamp(source // bs, max=tables.shape[1] - 1)) * bs + source % bs)[kept]
    target = (tables.gather(1, torch.clamp(target // bs, max=tables.shape[1] - 1)) * bs + target % bs)[kept]
    rows = _rows(st["pool"], case)
    rows[:, target] = rows[:, source]


def _run_plain(st):
    op = st["case"]["op"]
    if op == "append":
        st["q_out"].copy_(_rotate(st["q"].float(), st))
        _put(st, 0, _rotate(st["k"].float(), st))
        _put(st, 1, st["v"].float())
    elif op == "read":
        st["k_out"].copy_(_get(st, 0, st["slots"]))
        st["v_out"].copy_(_get(st, 1, st["slots"]))
    elif op == "attend":
        _attend_plain(st)
    else:
        _keep_plain(st)


def run(state):
    (_run_own if own else _run_plain)(state)
    case = state["case"]
    if case["op"] == "read":
        return {"k": state["k_out"], "v": state["v_out"]}
    if case["op"] == "attend":
        return {"out": state["out"], "lse": state["lse"]}
    cache = {"cache": _codes(state["pool"], case)}
    if case["fmt"] in LARGEST_CODE:
        cache["scales"] = _scales(state["pool"], case)
    return {"q": state["q_out"], **cache} if case["op"] == "append" else cache


# ---- the definition in 64 bits -----------------------------------------------------

def _values64(st, plane):
    """A plane of the cache in fp64, [slots][kv_heads][head_dim]."""
    case = st["case"]
    x = _codes(st["pool"], case)[plane].double()
    return x * _scales(st["pool"], case)[plane].double()[..., None] if case["fmt"] in LARGEST_CODE else x


def exact(case, seed):
    st = prepare(case, seed)
    op, d = case["op"], case["head_dim"]
    bs, h, hq = case["block_size"], case["kv_heads"], case["q_heads"]
    if op == "read":
        return {"k": _values64(st, 0)[st["slots"]], "v": _values64(st, 1)[st["slots"]]}
    if op == "append":
        # a pair of channels as a complex number, times exp(i * angle)
        rot = case["rot"]
        freq = 500000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=DEVICE) / rot)
        angle = st["positions"].double()[:, None] * freq
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]

        def turned(x):
            x = x.double().clone()
            first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["style"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            x[..., first], x[..., second] = z.real, z.imag
            return x

        rows = [turned(st["k"]), st["v"].double()]
        out = {"q": turned(st["q"])}
        if case["fmt"] in LARGEST_CODE:
            # the codes are rounded values; the scales and q have 64-bit ones
            scales = _scales(st["pool"], case).double()
            for plane, x in enumerate(rows):
                scales[plane][st["slots"]] = x.abs().amax(-1) / LARGEST_CODE[case["fmt"]]
            out.update(cache=None, scales=scales)
        else:
            out["cache"] = _codes(st["pool"], case).double()
            for plane, x in enumerate(rows):
                out["cache"][plane][st["slots"]] = x
        return out
    if op == "keep":
        return None                                                     # rows move as they are
    if sum(work(case).values()) > 2e12:
        return None
    out, lse = [], []
    context, new = _lengths(case)
    at = 0
    values = [_codes(st["pool"], case)[p] for p in (0, 1)]
    for r, (c, t) in enumerate(zip(context, new)):
        j = torch.arange(c + t, device=DEVICE)
        slots = st["tables"][r].long()[j // bs] * bs + j % bs
        kv = []
        for plane, x in enumerate(values):
            x = (x.view(torch.uint8)[slots].view(torch.float8_e4m3fn) if case["fmt"] == "e4m3" else x[slots]).double()
            if case["fmt"] in LARGEST_CODE:
                x = x * _scales(st["pool"], case)[plane][slots].double()[..., None]
            kv.append(x.transpose(0, 1))                                # [h, c + t, d]
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
