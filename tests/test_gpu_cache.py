"""The operators over the paged cache against plain implementations in 64 bits.

Error bounds, from the types alone (u16 = half a unit in the last place, relative: 2^-p for p bits of significand,
2^-8 for bf16, 2^-11 for f16):
  append, read, q_out  one rounding of an fp32 value: u16 |x|, plus 2^-22 max|x| for the fp32 products behind it
  e4m3 / int8          the decoded value is within half a step of the scale's grid: e4m3 2^-4 |x| + scale 2^-10, int8 scale / 2,
                       plus 2^-22 448 scale for the fp32 quotient
  attend               probabilities are rounded once (u16 of bf16, or of f16 where the product is f16) and so is the output:
                       |error| <= (u_p + u_out) A with A = sum_j p_j |v_j|, plus 2^-13 A for scores, exponentials and sums in
                       fp32 (|score| stays below 2^7 here: 2^7 2^-24 128 terms = 2^-10 would be the worst case of all signs
                       alike, the sum of 128 roundings at random is 2^-13.5), plus f16's subnormal steps: 2^-24 of the
                       largest |v| a key, and 2^-24 for the output
  lse                  2^-14 (1 + |lse|) by the same count
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

KIND = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
LARGEST = {"e4m3": 448.0, "int8": 127.0}


class Setup:
    """A cache, and requests with contexts `context` and `new` tokens each, blocks handed out at random."""

    def __init__(self, fmt, heads, dim, bs, context, new, layers=2, layout=0, seed=0, spare=3, poison=True):
        rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.fmt, self.heads, self.dim, self.bs, self.layers, self.layout = fmt, heads, dim, bs, layers, layout
        self.context, self.new = list(context), list(new)
        blocks = [-(-(c + t) // bs) for c, t in zip(context, new)]
        self.nb = sum(blocks) + spare
        self.cache = kvr.Cache(layers, heads, dim, bs, self.nb, fmt, layout)
        ids = rng.permutation(self.nb)[:sum(blocks)]
        width = max(blocks + [1]) + 1
        tables = rng.integers(0, self.nb, (len(blocks), width)).astype(np.int32)
        at = 0
        for r, n in enumerate(blocks):
            tables[r, :n] = ids[at:at + n]
            at += n
        self.host_tables = tables
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.starts, self.tokens = starts.tolist(), int(starts[-1])
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")          # noqa: E731
        self.arrays = (dev(starts), dev(context), dev(tables))
        self.batch = kvr.Batch(*self.arrays, max(new + [0]), max([c + t for c, t in zip(context, new)] + [0]), self.status)
        # every byte that no test writes is 0xff: NaN as bf16, f16, e4m3 and scales
        self.pool = torch.full((self.cache.pool_bytes,), 0xff if poison else 0, dtype=torch.uint8, device="cuda")

    def slot(self, r, j):
        return self.host_tables[r, j // self.bs] * self.bs + j % self.bs

    def slots(self, r, first, n):
        j = np.arange(first, first + n)
        return torch.from_numpy((self.host_tables[r, j // self.bs].astype(np.int64) * self.bs + j % self.bs)).cuda()

    def plane(self, layer, kv, pool=None):
        """One plane of a pool, [slots, row bytes] (a copy for block-major pools)."""
        pool = self.pool if pool is None else pool
        if self.layout == kvr.LAYER_MAJOR:
            return pool.view(self.layers, 2, self.nb * self.bs, -1)[layer, kv]
        return pool.view(self.nb, self.layers, 2, self.bs, -1)[:, layer, kv].reshape(self.nb * self.bs, -1)

    def decode(self, layer, kv, pool=None):
        """(values in fp64 [slots, heads, dim], scales or None)"""
        p = self.plane(layer, kv, pool).contiguous()
        n = self.heads * self.dim
        if self.fmt in ("bf16", "f16"):
            return p.view(KIND[self.fmt]).view(-1, self.heads, self.dim).double(), None
        kind = torch.float8_e4m3fn if self.fmt == "e4m3" else torch.int8
        codes = p[:, :n].contiguous().view(kind).view(-1, self.heads, self.dim).to(torch.float32).double()
        scales = p[:, n:n + 4 * self.heads].contiguous().view(torch.float32).double()
        return codes * scales[..., None], scales

    def fill(self, layer=0):
        """Valid tokens of every request through append, and what the cache then holds, [kv][request] in fp64."""
        lens = [c + t for c, t in zip(self.context, self.new)]
        starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        n = int(starts[-1])
        k, v = (torch.randn(n, self.heads, self.dim, device="cuda", generator=self.gen) for _ in range(2))
        k *= torch.exp(0.5 * torch.randn(self.heads, self.dim, device="cuda", generator=self.gen))
        v *= torch.exp(0.5 * torch.randn(n, 1, 1, device="cuda", generator=self.gen))
        whole = kvr.Batch(torch.from_numpy(starts).cuda(), torch.zeros_like(self.arrays[1]), self.arrays[2], max(lens + [0]), max(lens + [0]), self.status)
        if n:
            self.cache.append(self.pool, layer, whole, k=k, v=v)
        vals = [self.decode(layer, i)[0] for i in (0, 1)]
        return [[x[self.slots(r, 0, m)] for r, m in enumerate(lens)] for x in vals]

    def ok(self):
        torch.cuda.synchronize()
        assert int(self.status) == 0


def rand(s, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda", generator=s.gen).to(dtype)


def table_of(rot, positions, base=10000.0):
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def turn64(x, table, positions, rot, style, inverse=False):
    x = x.double().clone()
    cs = table.double()[positions.long()]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * (-1 if inverse else 1)
    i = torch.arange(rot // 2, device="cuda")
    a, b = (i, i + rot // 2) if style == "half" else (2 * i, 2 * i + 1)
    u, v = x[..., a].clone(), x[..., b].clone()
    x[..., a], x[..., b] = u * c - v * s, u * s + v * c
    return x


def assert_within(got, want, bound):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    bad = ((got - want).abs() > bound) & ~torch.isnan(want)
    assert not bad.any(), "%d of %d off, worst by %.3g of its bound" % (int(bad.sum()), bad.numel(), float(((got - want).abs() / bound).nan_to_num().max()))


# ---- append ------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["bf16", "f16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype,heads,q_heads,dim,rot,style,bs,layout", [
    ("bf16", 8, 32, 128, 128, "half", 16, 0), ("bf16", 2, 14, 64, 32, "interleaved", 5, 1), ("f16", 3, 9, 80, 20, "half", 1, 0),
    ("f32", 1, 1, 16, 6, "interleaved", 7, 0), ("f16", 5, 5, 256, 256, "half", 16, 1), ("f32", 9, 18, 112, 96, "half", 8, 0),
    ("bf16", 4, 4, 144, 2, "half", 32, 0)])
def test_append_matches_the_formula_and_touches_nothing_else(fmt, dtype, heads, q_heads, dim, rot, style, bs, layout):
    s = Setup(fmt, heads, dim, bs, [0, 37, 5, 0, 64], [1, 3, 0, 19, 130], layout=layout, seed=dim + heads)
    kind = KIND[dtype]
    wide = rand(s, s.tokens, q_heads + 2 * heads, dim, dtype=kind)                # q, k, v side by side
    q, k, v = wide[:, :q_heads], wide[:, q_heads:q_heads + heads], wide[:, q_heads + heads:]
    pos = torch.randint(0, 500, (s.tokens,), device="cuda", generator=s.gen, dtype=torch.int32)
    table = table_of(rot, 500)
    q_out = torch.full((q_heads, s.tokens, dim), 7.0, dtype=kind, device="cuda").transpose(0, 1)    # heads outermost
    before = s.pool.clone()
    s.cache.append(s.pool, 1, s.batch, q=q, k=k, v=v, q_out=q_out, rope=kvr.Rope(table, rot, style), positions=pos)
    s.ok()
    want_q = turn64(q, table, pos, rot, style)
    assert_within(q_out, want_q, U[dtype] * want_q.abs() + 2.0 ** -22 * 8)
    written = torch.cat([s.slots(r, c, t) for r, (c, t) in enumerate(zip(s.context, s.new))])
    for kv, x in ((0, turn64(k, table, pos, rot, style)), (1, v.double())):
        got, scales = s.decode(1, kv)
        got = got[written]
        if fmt in LARGEST:
            want_s = x.abs().amax(-1) / LARGEST[fmt]
            assert_within(scales[written], want_s, 2.0 ** -21 * want_s)
            step = want_s[..., None]
            half = step / 2 if fmt == "int8" else 2.0 ** -4 * x.abs() + step * 2.0 ** -10
            assert_within(got, x, half + 2.0 ** -20 * 448 * step)
        else:
            assert_within(got, x, U[fmt] * x.abs() + 2.0 ** -22 * 8 + (2.0 ** -25 if fmt == "f16" else 0))
    # all other rows of all planes are as they were
    for layer in range(2):
        for kv in range(2):
            a, b = s.plane(layer, kv).clone(), s.plane(layer, kv, before).clone()
            if layer == 1:
                a[written] = 0
                b[written] = 0
            assert torch.equal(a, b)


def test_append_in_place_inverse_and_default_positions():
    s = Setup("bf16", 2, 96, 16, [3, 0], [40, 9], seed=5)
    for rot, style in ((96, "half"), (20, "half"), (22, "interleaved")):
        table = table_of(rot, 64)
        pos = torch.cat([torch.arange(3, 43), torch.arange(9)]).int().cuda()
        x = rand(s, s.tokens, 6, 96, dtype=torch.float32)
        y = x.clone()
        s.cache.append(s.pool, 0, s.batch, q=y, q_out=y, rope=kvr.Rope(table, rot, style))           # q alone, in place
        want = turn64(x, table, pos, rot, style)
        assert_within(y, want, 2.0 ** -22 * 8 + 0 * want)
        s.cache.append(s.pool, 0, s.batch, q=y, q_out=y, rope=kvr.Rope(table, rot, style, inverse=True), positions=pos)
        assert_within(y, x, 2.0 ** -20 * 8 + 0 * want)
    s.ok()


def test_append_without_rope_k_or_v_alone():
    s = Setup("f16", 3, 64, 4, [2], [9], seed=6)
    k = rand(s, 9, 3, 64, dtype=torch.float16)
    before = s.pool.clone()
    s.cache.append(s.pool, 0, s.batch, k=k)
    s.ok()
    assert torch.equal(s.decode(0, 0)[0][s.slots(0, 2, 9)], k.double())
    assert torch.equal(s.plane(0, 1), s.plane(0, 1, before))
    s.cache.append(s.pool, 0, s.batch, v=k)
    assert torch.equal(s.decode(0, 1)[0][s.slots(0, 2, 9)], k.double())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_quantising_odd_values(fmt):
    """Zeros, subnormals, the largest numbers, and what is not finite."""
    s = Setup(fmt, 4, 32, 16, [0], [6])
    x = torch.zeros(6, 4, 32, device="cuda")
    x[1] = 1e-40
    x[1, :, 0] = 1.1754944e-38
    big = torch.finfo(torch.float32).max
    x[2, :, 3], x[2, :, 4] = big, -big
    x[3, 1, 5], x[3, 2, 6], x[3, 3, 31] = math.inf, -math.inf, math.nan
    x[3, 0] = 1.0
    x[4] = torch.linspace(-1, 1, 32, device="cuda")
    x[5, :, 7] = -1e-30
    s.cache.append(s.pool, 0, s.batch, k=x, v=x)
    out = torch.zeros(6, 4, 32, device="cuda")
    s.cache.read(s.pool, 0, s.batch, k=out)
    s.ok()
    assert (out[0] == 0).all()
    assert (out[1] - x[1]).abs().max() <= 2.0 ** -126 * 0.5 and torch.isfinite(out[1]).all()
    assert torch.isfinite(out[2]).all() and (out[2, :, 3] - x[2, :, 3]).abs().max() <= 2.0 ** -21 * 3.5e38
    assert torch.isnan(out[3, 1:]).all() and (out[3, 0] == 1).all()
    assert_within(out[4], x[4].double(), 0.5 / 127 + 2.0 ** -4 * x[4].abs().double())
    assert (out[5, :, 7] + 1e-30).abs().max() <= 2.0 ** -21 * 1e-30 and (out[5, :, :7] == 0).all()


def test_scaled_tables():
    for kw in (dict(kind=kvr.SCALE_BANDS, base=500000.0, factor=8.0, low=1.0, high=4.0, original=8192),
               dict(kind=kvr.SCALE_RAMP, base=10000.0, factor=16.0, low=1.0, high=32.0, original=4096), dict(base=10000.0)):
        f, m = kvr.rope_frequencies(128, **kw)
        out = torch.empty(700, 64, 2, device="cuda")
        kvr.rope_table(out, first=1000000, **kw)
        a = torch.arange(1000000, 1000700, dtype=torch.float64, device="cuda")[:, None] * torch.from_numpy(f).cuda()
        # one rounding to fp32, and the fp64 angle's own (2^20 2^-53)
        assert_within(out, torch.stack([a.cos(), a.sin()], -1) * m, 2.0 ** -24 * m + 2.0 ** -30)


# ---- read --------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["bf16", "f16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype,heads,dim,bs,layout", [("bf16", 8, 128, 16, 0), ("f16", 2, 64, 5, 1), ("f32", 3, 80, 1, 0), ("bf16", 1, 256, 8, 0), ("f32", 9, 16, 3, 1)])
def test_read_returns_what_the_cache_holds(fmt, dtype, heads, dim, bs, layout):
    s = Setup(fmt, heads, dim, bs, [0, 7, 0, 33], [21, 40, 0, 1], layout=layout, seed=dim)
    k, v = s.fill(1)
    wide = torch.full((s.tokens, heads + 1, dim + 16), 5.0, dtype=KIND[dtype], device="cuda")
    k_out, v_out = wide[:, :heads, :dim], torch.zeros(heads, s.tokens, dim, dtype=KIND[dtype], device="cuda").transpose(0, 1)
    s.cache.read(s.pool, 1, s.batch, k=k_out, v=v_out)
    s.ok()
    for got, want in ((k_out, k), (v_out, v)):
        want = torch.cat([w[c:] for w, c in zip(want, s.context)])
        tiny = 2.0 ** -25 if dtype == "f16" else 0
        assert_within(got, want, (U[dtype] + 2.0 ** -24) * want.abs() + tiny)
    assert (wide[:, heads] == 5).all() and (wide[..., dim:] == 5).all()
    only = torch.zeros(s.tokens, heads, dim, dtype=KIND[dtype], device="cuda")
    s.cache.read(s.pool, 1, s.batch, v=only)
    assert torch.equal(only, v_out.contiguous())


# ---- attend ------------------------------------------------------------------------

def attend64(s, q, k, v, scale, seen):
    """out, lse and A = sum p |v| of the definition; seen[r]: [new, context + new]."""
    out, lse, mag = [], [], []
    g = q.shape[1] // s.heads
    for r, (c, t) in enumerate(zip(s.context, s.new)):
        if t == 0:
            continue
        x = q[s.starts[r]:s.starts[r] + t].double().view(t, s.heads, g, s.dim)
        sc = torch.einsum("thgd,jhd->thgj", x, torch.where(seen[r].any(0)[:, None, None], k[r], 0.0)) * scale
        # what a row does not see has no part in its sums, whatever it is
        sc = torch.where(seen[r][:, None, None], sc, -math.inf)
        m = sc.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)
        p = torch.exp(sc - m)
        l = p.sum(-1, keepdim=True)
        p = torch.where(l > 0, p / l, 0.0)
        o = torch.zeros(t, s.heads, g, s.dim, dtype=torch.float64, device="cuda")
        a = torch.zeros_like(o)
        finite = torch.isfinite(v[r])
        o += torch.einsum("thgj,jhd->thgd", p, torch.where(finite, v[r], 0.0))
        a += torch.einsum("thgj,jhd->thgd", p, torch.where(finite, v[r], 0.0).abs())
        for j in torch.nonzero(~finite.all(-1).all(-1))[:, 0].tolist():              # one key at a time
            rows = seen[r][:, j]
            bad = torch.where(finite[j], 0.0, v[r][j])[None, :, None].expand(int(rows.sum()), -1, g, -1)
            o[rows] += bad
        out.append(o.reshape(t, q.shape[1], s.dim))
        mag.append(a.reshape(t, q.shape[1], s.dim))
        lse.append((m + torch.log(l))[..., 0].reshape(t, q.shape[1]))
    return torch.cat(out), torch.cat(lse), torch.cat(mag)


def causal(s):
    out = []
    for c, t in zip(s.context, s.new):
        m = torch.ones(t, c + t, dtype=torch.bool, device="cuda")
        m[:, c:] = torch.ones(t, t, dtype=torch.bool, device="cuda").tril()
        out.append(m)
    return out


def tree(s, rng, empty=0.0, context_too=True):
    """Random trees (any earlier node as parent) as bit words, and the same as truth values."""
    words = max(1, -(-max(s.new) // 64))
    bits = np.zeros((s.tokens, words * 64), dtype=bool)
    seen = []
    for r, (c, t) in enumerate(zip(s.context, s.new)):
        rows = bits[s.starts[r]:s.starts[r] + t]
        for i in range(t):
            if i and rng.random() < 0.9:
                rows[i] = rows[int(rng.integers(0, i))]
            rows[i, i] = True
        rows[rng.random(t) < empty] = False
        m = torch.ones(t, c + t, dtype=torch.bool, device="cuda")
        m[:, c:] = torch.from_numpy(rows[:, :t].copy()).cuda()
        seen.append(m)
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int64)).cuda(), seen


def check_attend(s, q_heads, dtype, mask=None, seen=None, scale=None, layer=0, strided=False, kv=None):
    kind = KIND[dtype]
    k, v = s.fill(layer) if kv is None else kv
    scale = 1 / math.sqrt(s.dim) if scale is None else scale
    if strided:
        q = rand(s, s.tokens, q_heads + 2, s.dim + 8, dtype=kind)[:, 1:-1, :s.dim]
        q = torch.empty(q_heads, s.tokens, s.dim, dtype=kind, device="cuda").transpose(0, 1).copy_(q)
        out = torch.full((s.tokens, q_heads + 1, s.dim), 9.0, dtype=kind, device="cuda")[:, :-1]
    else:
        q, out = rand(s, s.tokens, q_heads, s.dim, dtype=kind), torch.full((s.tokens, q_heads, s.dim), 9.0, dtype=kind, device="cuda")
    lse = torch.full((s.tokens, q_heads), 9.0, device="cuda")
    ws = torch.full((s.cache.workspace_bytes(),), 0xff, dtype=torch.uint8, device="cuda")           # of no interest, but for
    ws[:4096] = 0                                                                                    # the counters
    s.cache.attend(s.pool, layer, s.batch, q, out, ws, lse=lse, mask=mask, scale=scale)
    s.ok()
    want, want_lse, mag = attend64(s, q, k, v, scale, causal(s) if seen is None else seen)
    u_p = U["bf16"] if s.fmt == "bf16" else U["f16"]
    top = max([float(torch.nan_to_num(x, 0, 0, 0).abs().max()) for x in v if x.numel()] + [0.0])
    keys = max(c + t for c, t in zip(s.context, s.new))
    tiny = 0 if s.fmt == "bf16" else 2.0 ** -24 * top * math.sqrt(keys)
    assert_within(out, want, (u_p + U[dtype] + 2.0 ** -13) * mag + tiny + (2.0 ** -24 if dtype == "f16" else 2.0 ** -100))
    some = want_lse != -math.inf
    assert torch.equal(some, lse != -math.inf)
    assert_within(lse[some], want_lse[some], 2.0 ** -14 * (1 + want_lse[some].abs()))
    again = torch.zeros_like(out)
    s.cache.attend(s.pool, layer, s.batch, q, again, ws, mask=mask, scale=scale)                     # no lse; the same bits
    assert torch.equal(again.view(torch.int16), out.contiguous().view(torch.int16))
    assert not ws[:4096].any()
    return out, lse, q


DIMS = [(8, 4, 128, 16), (2, 8, 128, 16), (1, 1, 64, 8), (3, 5, 80, 5), (4, 2, 256, 16), (12, 1, 64, 16), (5, 3, 96, 7), (8, 7, 64, 32), (1, 16, 192, 1)]


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16"), ("e4m3", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("heads,group,dim,bs", DIMS)
def test_attend_single_tokens(fmt, dtype, heads, group, dim, bs):
    """One new token a request, contexts from none to thousands of tokens."""
    s = Setup(fmt, heads, dim, bs, [0, 1, 14, 15, 16, 17, 63, 64, 255, 700, 3001], [1] * 11, seed=heads * dim)
    check_attend(s, heads * group, dtype)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("heads,group,dim,bs", DIMS)
def test_attend_trees_with_empty_rows(fmt, dtype, heads, group, dim, bs):
    """Trees of up to 70 tokens (two mask words); rows that see nothing at all where there is no context."""
    s = Setup(fmt, heads, dim, bs, [0, 0, 100, 511, 1000, 33, 0], [1, 7, 13, 64, 70, 0, 70], seed=heads * dim + 1, layout=heads % 2)
    mask, seen = tree(s, np.random.default_rng(dim), empty=0.15)
    out, lse, _ = check_attend(s, heads * group, dtype, mask, seen, strided=True)
    empty = torch.cat([~m.any(1) for m in seen])
    assert empty.any() and (out[empty] == 0).all() and (lse[empty] == -math.inf).all()


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "bf16")])
def test_attend_causal_chunks(fmt, dtype):
    """Without a mask the new tokens see each other in order; a chunk longer than any tile."""
    s = Setup(fmt, 2, 128, 16, [0, 300, 5], [200, 129, 1], seed=3)
    check_attend(s, 8, dtype)


@pytest.mark.parametrize("new", [2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65])
@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("e4m3", "bf16")])
def test_attend_every_tile_of_rows(fmt, dtype, new):
    s = Setup(fmt, 2, 128, 16, [129, 40], [new, max(1, new // 2)], seed=new)
    mask, seen = tree(s, np.random.default_rng(new))
    check_attend(s, 8, dtype, mask, seen)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("group", [1, 8])
def test_attend_ignores_what_a_row_does_not_see(fmt, dtype, group):
    """K and V of some drafted tokens are NaN, infinite or the type's lowest number; rows that do not see them are as if
    they were not there, rows that do are the formula's."""
    s = Setup(fmt, 2, 64, 16, [0, 50, 200], [9, 20, 33], seed=11)
    mask, seen = tree(s, np.random.default_rng(4))
    k, v = s.fill()
    odd = {1: math.nan, 3: math.inf, 6: -math.inf, 7: -6e4}
    for r, (c, t) in enumerate(zip(s.context, s.new)):
        for j, value in odd.items():
            one = kvr.Batch(torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([c + j], dtype=torch.int32, device="cuda"),
                            s.arrays[2][r:r + 1].contiguous(), 1, c + t, s.status)
            x = torch.ones(1, 2, 64, device="cuda", dtype=torch.float32)
            x[0, 1, 5] = value
            s.cache.append(s.pool, 0, one, v=x)
            if j != 7 and value != value:
                s.cache.append(s.pool, 0, one, k=x)
    vals = [s.decode(0, i)[0] for i in (0, 1)]
    kv = [[x[s.slots(r, 0, c + t)] for r, (c, t) in enumerate(zip(s.context, s.new))] for x in vals]
    q = rand(s, s.tokens, 2 * group, 64, dtype=KIND[dtype])
    out, lse, ws = torch.zeros_like(q), torch.zeros(s.tokens, 2 * group, device="cuda"), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    s.cache.attend(s.pool, 0, s.batch, q, out, ws, lse=lse, mask=mask)
    s.ok()
    at = 0
    for r, (c, t) in enumerate(zip(s.context, s.new)):
        clean = ~seen[r][:, [c + j for j in odd if j < t]].any(1)
        assert clean.any()
        # the same with the odd tokens' rows set to something tame
        for i in torch.nonzero(clean)[:, 0].tolist():
            keys = torch.nonzero(seen[r][i])[:, 0]
            for h in range(2):
                kk, vv = kv[0][r][keys, h], kv[1][r][keys, h]
                for g in range(group):
                    sc = kk @ q[at + i, h * group + g].double() / 8.0
                    p = torch.softmax(sc, 0)
                    bound = (U["bf16"] + U[dtype] + 2.0 ** -13) * (p @ vv.abs()) + 2.0 ** -12
                    assert_within(out[at + i, h * group + g], p @ vv, bound)
        hit = seen[r][:, c + 1]
        assert torch.isnan(out[at:at + t][hit][:, group:, 5]).all()                 # NaN in K and V of a token it sees
        if fmt in ("bf16", "f16"):
            other = (seen[r][:, c + 3] & ~seen[r][:, c + 1] & ~seen[r][:, c + 6])
            assert (out[at:at + t][other][:, group:, 5] == math.inf).all()
            assert torch.isfinite(out[at:at + t][other][:, group:, 6]).all()        # other channels of that token are numbers
        at += t


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("new", [1, 40])
def test_attend_large_and_unlike_values(fmt, dtype, new):
    """Scores far apart (the running maximum moves late and far), values of V across many magnitudes."""
    s = Setup(fmt, 2, 128, 16, [900, 64], [new, new], seed=21, poison=False)
    k, v = s.fill()
    lens = [c + t for c, t in zip(s.context, s.new)]
    starts = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
    whole = kvr.Batch(starts, torch.zeros_like(s.arrays[1]), s.arrays[2], max(lens), max(lens), s.status)
    n = sum(lens)
    ramp = torch.linspace(0.1, 3.0, n, device="cuda")[:, None, None]
    kk = rand(s, n, 2, 128, dtype=torch.float32) * ramp
    vv = rand(s, n, 2, 128, dtype=torch.float32) * torch.exp2(torch.randint(-6, 7, (n, 2, 1), device="cuda", generator=s.gen).float())
    s.cache.append(s.pool, 0, whole, k=kk, v=vv)
    vals = [s.decode(0, i)[0] for i in (0, 1)]
    kv = [[x[s.slots(r, 0, m)] for r, m in enumerate(lens)] for x in vals]
    check_attend(s, 8, dtype, scale=0.5, kv=kv)


def test_attend_small_values_of_v():
    """V's scales far from one, in both directions."""
    for size in (1e-30, 1e-6, 1e6, 1e30):
        for new in (1, 40):
            s = Setup("e4m3", 2, 64, 16, [200], [new], seed=22)
            n = 200 + new
            whole = kvr.Batch(torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.zeros_like(s.arrays[1]), s.arrays[2], n, n, s.status)
            k, v = rand(s, n, 2, 64, dtype=torch.float32), rand(s, n, 2, 64, dtype=torch.float32)
            s.cache.append(s.pool, 0, whole, k=k, v=v * size)
            kv = [[s.decode(0, i)[0][s.slots(0, 0, n)]] for i in (0, 1)]
            q, ws = rand(s, new, 4, 64), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
            out = torch.zeros(new, 4, 64, dtype=torch.bfloat16, device="cuda")
            s.cache.attend(s.pool, 0, s.batch, q, out, ws)
            s.ok()
            want, _, mag = attend64(s, q, *kv, 1 / 8.0, causal(s))
            assert_within(out, want, (U["f16"] + U["bf16"] + 2.0 ** -13) * mag + 2.0 ** -24 * 8 * size * 16)


def test_attend_zero_rows_of_v_and_k():
    s = Setup("int8", 1, 64, 16, [40], [1], seed=23)
    whole = kvr.Batch(torch.tensor([0, 41], dtype=torch.int32, device="cuda"), torch.zeros_like(s.arrays[1]), s.arrays[2], 41, 41, s.status)
    k, v = torch.zeros(41, 1, 64, device="cuda"), torch.zeros(41, 1, 64, device="cuda")
    s.cache.append(s.pool, 0, whole, k=k, v=v)
    q, out = rand(s, 1, 4, 64), torch.ones(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    lse, ws = torch.zeros(1, 4, device="cuda"), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    s.cache.attend(s.pool, 0, s.batch, q, out, ws, lse=lse)
    s.ok()
    assert (out == 0).all() and (lse - math.log(41)).abs().max() < 1e-5


@pytest.mark.parametrize("new,heads", [(1, 8), (33, 8), (1, 1)])
def test_attend_many_requests_and_many_pieces(new, heads):
    """More requests than threads of a CTA, most of them short; and one request cut into as many pieces as there are SMs."""
    rng = np.random.default_rng(1)
    n = 600 if new == 1 else 40
    s = Setup("bf16", heads, 64, 16, [int(x) for x in rng.integers(0, 40, n)], [new] * n, seed=31)
    check_attend(s, heads * 2, "bf16")
    s = Setup("bf16", heads, 64, 16, [20000], [new], seed=32)
    check_attend(s, heads * 2, "bf16")
    if new > 1:
        s = Setup("bf16", heads, 64, 16, [3, 5, 20000, 0], [0, new, new, 0], seed=33)
        mask, seen = tree(s, rng)
        check_attend(s, heads * 2, "bf16", mask, seen)


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_offsets_beyond_32_bits(fmt):
    """Blocks behind the first 4 GiB of a plane, and a layer behind them."""
    heads, dim, bs = 8, 128, 16
    row = 2048 if fmt == "bf16" else 1056
    s = Setup(fmt, heads, dim, bs, [100, 30], [20, 1], layers=1, spare=(5 << 30) // (row * bs), seed=41, poison=False)
    # the last blocks of the pool
    width = s.host_tables.shape[1]
    s.host_tables[:] = (s.nb - 1 - np.arange(2 * width).reshape(2, width)).astype(np.int32)
    s.arrays[2].copy_(torch.from_numpy(s.host_tables))
    n = 151
    k, v = (rand(s, n, heads, dim) for _ in range(2))
    whole = kvr.Batch(torch.tensor([0, 120, 151], dtype=torch.int32, device="cuda"), torch.zeros_like(s.arrays[1]), s.arrays[2], 120, 120, s.status)
    table = table_of(dim, 200)
    s.cache.append(s.pool, 0, whole, k=k, v=v, rope=kvr.Rope(table, dim))
    out = torch.zeros(n, heads, dim, device="cuda")
    s.cache.read(s.pool, 0, whole, k=out)
    pos = torch.cat([torch.arange(120), torch.arange(31)]).cuda()
    want = turn64(k, table, pos, dim, "half")
    step = want.abs().amax(-1, keepdim=True) / 127
    assert_within(out, want, U["bf16"] * want.abs() + 1e-5 if fmt == "bf16" else step * 0.51)
    got = [torch.zeros(n, heads, dim, device="cuda") for _ in range(2)]
    s.cache.read(s.pool, 0, whole, k=got[0], v=got[1])
    kv = [[x[:120].double(), x[120:].double()] for x in got]
    check_attend(s, 32, "bf16", kv=kv)


def test_what_does_not_fit_is_left_out_and_reported():
    for what in ("block", "new", "tokens", "table", "start"):
        s = Setup("bf16", 2, 64, 16, [20, 20, 20], [2, 2, 2], seed=51)
        s.fill()
        starts, context, tables = (x.clone() for x in s.arrays)
        max_new, max_tokens = 2, 22
        if what == "block":
            tables[1, 1] = s.nb
        elif what == "new":
            max_new = 1
        elif what == "tokens":
            context[1] = 21
        elif what == "table":
            max_tokens, context[1] = 10 ** 6, 16 * tables.shape[1] - 1
        else:
            starts[2] = 1
        b = kvr.Batch(starts, context, tables, max_new, max_tokens, s.status)
        q, out = rand(s, 6, 4, 64), torch.full((6, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        code = kvr.DEV_BAD_BLOCK if what == "block" else kvr.DEV_BAD_LENGTH
        before = s.pool.clone()
        s.cache.attend(s.pool, 0, b, q, out, ws)
        torch.cuda.synchronize()
        assert int(s.status) == code, what
        if what in ("tokens", "table"):
            assert (out[2:4] == 3).all() and (out[:2] != 3).any() and (out[4:] != 3).any()
        s.status.zero_()
        s.cache.read(s.pool, 0, b, k=torch.zeros(6, 2, 64, device="cuda"))
        torch.cuda.synchronize()
        assert int(s.status) == code
        s.status.zero_()
        s.cache.append(s.pool, 0, b, k=rand(s, 6, 2, 64))
        torch.cuda.synchronize()
        assert int(s.status) == code
        if what == "block":                      # the two tokens of request 1 lie in the bad block: nothing of them is written
            rest = [int(s.slot(r, j)) for r in (0, 2) for j in (20, 21)]
            a, c = s.plane(0, 0).clone(), s.plane(0, 0, before).clone()
            a[rest] = 0
            c[rest] = 0
            assert torch.equal(a, c)
        s.status.zero_()
        s.cache.keep(s.pool, b, torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert int(s.status) == code
    s = Setup("bf16", 2, 64, 16, [20], [2], seed=52)
    y = rand(s, 2, 2, 64)
    out = torch.full_like(y, 3.0)
    s.cache.append(s.pool, 0, s.batch, q=y, q_out=out, rope=kvr.Rope(table_of(64, 21), 64))               # positions 20 and 21 of 21
    torch.cuda.synchronize()
    assert int(s.status) == kvr.DEV_BAD_POSITION and (out[1] == 3).all() and (out[0] != 3).any()


# ---- keep --------------------------------------------------------------------------

@pytest.mark.parametrize("fmt,heads,dim,bs,layers,layout", [("bf16", 8, 128, 16, 3, 0), ("e4m3", 3, 48, 5, 2, 1), ("int8", 8, 128, 16, 4, 0), ("f16", 1, 16, 1, 1, 1)])
def test_keep_moves_accepted_rows(fmt, heads, dim, bs, layers, layout):
    s = Setup(fmt, heads, dim, bs, [0, 15, 16, 100, 7, 3], [1, 20, 70, 200, 0, 5], layers=layers, layout=layout, seed=bs)
    s.pool.random_(0, 256, generator=s.gen)
    lists = [[0], [0, 3, 4, 19], list(range(70)), sorted(np.random.default_rng(2).permutation(200)[:150].tolist()), [], []]
    index = torch.zeros(6, 160, dtype=torch.int32)
    for r, x in enumerate(lists):
        index[r, :len(x)] = torch.tensor(x, dtype=torch.int32)
    before = s.pool.clone()
    s.cache.keep(s.pool, s.batch, index.cuda(), torch.tensor([len(x) for x in lists], dtype=torch.int32, device="cuda"))
    s.ok()
    for layer in range(layers):
        for kv in range(2):
            want = s.plane(layer, kv, before).clone()
            old = want.clone()
            for r, x in enumerate(lists):
                for i, j in enumerate(x):
                    want[s.slot(r, s.context[r] + i)] = old[s.slot(r, s.context[r] + j)]
            assert torch.equal(s.plane(layer, kv), want)


def test_keep_refuses_lists_on_the_device():
    for row, n in (([1, 1], 2), ([2, 1], 2), ([0, 4], 2), ([-1, 0], 2), ([0, 1], 5), ([0, 1], -1), ([0, 1], 3)):
        s = Setup("bf16", 2, 64, 16, [10, 10], [4, 4], seed=61)
        s.pool.random_(0, 256, generator=s.gen)
        before = s.pool.clone()
        index = torch.tensor([row, [1, 3]], dtype=torch.int32, device="cuda")
        s.cache.keep(s.pool, s.batch, index, torch.tensor([n, 2], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert int(s.status) == kvr.DEV_BAD_INDEX
        # the other request's rows moved, this one's did not
        a, b = s.plane(0, 0).clone(), s.plane(0, 0, before).clone()
        b[[s.slot(1, 10), s.slot(1, 11)]] = b[[s.slot(1, 11), s.slot(1, 13)]]
        assert torch.equal(a, b), (row, n)


# ---- together ----------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_a_step_on_another_stream_and_in_a_graph(fmt):
    """append -> attend -> keep captured once on a side stream and replayed with other lengths in the same arrays."""
    s = Setup(fmt, 2, 64, 16, [100, 64], [6, 6], layers=1, seed=71)
    k, v = s.fill()
    mask, seen = tree(s, np.random.default_rng(3))
    q, kn, vn = rand(s, 12, 8, 64), rand(s, 12, 2, 64), rand(s, 12, 2, 64)
    out, ws = torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    index, count = torch.tensor([[0, 2], [1, 5]], dtype=torch.int32, device="cuda"), torch.tensor([2, 2], dtype=torch.int32, device="cuda")
    table = table_of(64, 200)
    b = kvr.Batch(*s.arrays, 6, 106, s.status)

    def step():
        s.cache.append(s.pool, 0, b, q=q, k=kn, v=vn, q_out=q, rope=kvr.Rope(table, 64))
        s.cache.attend(s.pool, 0, b, q, out, ws, mask=mask)
        s.cache.keep(s.pool, b, index, count)

    start_pool, start_q, side = s.pool.clone(), q.clone(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    first, pool_after = out.clone(), s.pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ([100, 64], [41, 50]):
        s.pool.copy_(start_pool)
        q.copy_(start_q)
        s.arrays[1].copy_(torch.tensor(lengths, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        if lengths == [100, 64]:
            assert torch.equal(out, first) and torch.equal(s.pool, pool_after)
        else:
            replayed = out.clone()
            s.pool.copy_(start_pool)
            q.copy_(start_q)
            step()
            torch.cuda.synchronize()
            assert torch.equal(out, replayed) and not torch.equal(out, first)
    assert int(s.status) == 0


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_attention_survives_a_suspend_and_resume(fmt):
    """The pool's movers carry codes and scales: the answer after a resume into other blocks is the same, bit for bit."""
    c = kvr.Cache(2, 4, 64, 16, 200, fmt)
    pool = torch.zeros(c.pool_bytes, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, new = 500, 5
    with kvr.Pool(*c.geometry, 200, 64 << 20, initial_free_order=np.random.default_rng(1).permutation(200).astype(np.int32),
                  device_pool=pool.data_ptr()) as p:
        assert c.pool_bytes == 200 * 16 * kvr.bytes_per_token(*c.geometry[:4])
        st, blocks = p.admit(1, n)
        assert st == kvr.OK
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")       # noqa: E731
        k, v, q = (torch.randn(n, h, 64, device="cuda", generator=gen).bfloat16() for h in (4, 4, 8))
        for layer in range(2):
            c.append(pool, layer, kvr.Batch(i32([0, n]), i32([0]), i32(blocks)[None], n, n), k=k, v=v)
        ws = torch.zeros(c.workspace_bytes(), dtype=torch.uint8, device="cuda")
        answers = []
        for _ in range(2):
            st, d = p.info(1)
            out = torch.zeros(2, new, 8, 64, dtype=torch.bfloat16, device="cuda")
            for layer in range(2):
                c.attend(pool, layer, kvr.Batch(i32([0, new]), i32([n - new]), i32(d["blocks"])[None], new, n), q[:new], out[layer], ws)
            torch.cuda.synchronize()
            answers.append((d["blocks"].tolist(), out))
            if len(answers) == 1:
                assert p.suspend_to_host([1], kvr.SYNC)[0] == kvr.OK
                assert p.stats()["bytes_suspended"] == n * kvr.bytes_per_token(*c.geometry[:4])
                pool.fill_(0xff)
                assert p.resume_from_host([1], kvr.SYNC)[0] == kvr.OK
        assert answers[0][0] != answers[1][0] and torch.equal(answers[0][1], answers[1][1])
