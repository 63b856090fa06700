"""A cache held in 4 bits, positions with several axes and copies of blocks, against plain implementations.

Error bounds, from the types alone (a rounding is off by at most half a step, eps / 2):
  append to 4 bits   codes, groups' scales and scales are the header's formulas in fp32, one rounding after the other, so the bytes are
                     those of the same steps in torch.  By value: a code is off by at most half of the largest step (1 of 2, at 4 to 6), and what the
                     group's scale pushed past 6 stays there: g is rounded, by 2^-4, so at most 6 (1 + 2^-4) became 6: within (1 + 2^-10) g S of the element; where
                     g is subnormal (below 2^-6) its half step is 2^-10, an element of 6 of those becomes at least 0, at most 6 g: within 7 2^-10 S
  read               code times g is exact, times S one rounding, the output's type another
  attend             as in test_gpu_cache.py for caches whose products are f16: code times g is exact in f16
"""
import math

import numpy as np
import pytest
import torch

import test_gpu_cache as base
from paper_2608_30830_b200 import kvr
from test_gpu_cache import KIND, U, assert_within, rand, table_of, turn64

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def records(s, layer, kv, pool=None):
    """A plane's records, [slots, heads, bytes]."""
    return s.plane(layer, kv, pool).contiguous().unflatten(-1, (s.heads, -1))


class Setup(base.Setup):
    def decode(self, layer, kv, pool=None):
        if self.fmt != "e2m1":
            return super().decode(layer, kv, pool)
        r, d = records(self, layer, kv, pool), self.dim
        codes = torch.stack([r[..., :d // 2] & 15, r[..., :d // 2] >> 4], -1).flatten(-2)
        scale = r[..., d // 2:d // 2 + 4].contiguous().view(torch.float32)[..., 0].double()
        byte = (r[..., d // 2 + 4:d // 2 + 4 + d // 16] & 0x7f).contiguous()
        group = torch.where(byte == 0x7f, 480.0, byte.view(torch.float8_e4m3fn).float().double())
        return (VALUES.cuda()[codes.int()].unflatten(-1, (-1, 16)) * group[..., None]).flatten(-2) * scale[..., None], scale


def pack(x):
    """The records' bytes of x [..., dim] in fp32, by the header's steps."""
    d = x.shape[-1]
    c = lambda v: torch.tensor(v, dtype=torch.float32, device=x.device)                    # noqa: E731
    g = x.unflatten(-1, (-1, 16))
    finite = torch.isfinite(x).all(-1, keepdim=True)
    scale = torch.clamp(x.abs().amax(-1, keepdim=True) * c(1 / 2688), min=2.0 ** -100)
    group = torch.clamp(g.abs().amax(-1) * ((c(1.0) / scale) * c(1 / 6)), max=448.0)
    group = torch.where(finite, group, 0.0).to(torch.float8_e4m3fn)
    step = group.float() * scale
    y = g * torch.where(group.float() > 0, c(1.0) / step, 0.0)[..., None]
    a = y.abs()
    code = torch.where(a <= 2, (a * 2).round(), torch.where(a <= 4, a.round() + 2, torch.clamp((a / 2).round() + 4, max=7)))
    code = (code.nan_to_num().to(torch.uint8) | torch.signbit(y).to(torch.uint8) << 3).flatten(-2)
    code = torch.where(finite, code, torch.zeros_like(code))
    out = torch.zeros(x.shape[:-1] + (-(-(d // 2 + 4 + d // 16) // 16) * 16,), dtype=torch.uint8, device=x.device)
    out[..., :d // 2] = code[..., 0::2] | code[..., 1::2] << 4
    scale = torch.where(finite, scale, torch.tensor(math.nan, device=x.device))
    out[..., d // 2:d // 2 + 4] = scale.contiguous().view(torch.uint8)
    out[..., d // 2 + 4:d // 2 + 4 + d // 16] = group.view(torch.uint8)
    return out


def same_records(got, want, d):
    """Byte for byte, but for which NaN stands for the scale of a head that is not finite."""
    got, want = got.clone(), want.clone()
    for x in (got, want):
        scale = x[..., d // 2:d // 2 + 4].contiguous().view(torch.float32)
        scale[torch.isnan(scale)] = -1.0
        x[..., d // 2:d // 2 + 4] = scale.view(torch.uint8)
    assert torch.equal(got, want), "%d bytes differ" % int((got != want).sum())


# ---- append and read ---------------------------------------------------------------

SHAPES = [("bf16", 8, 32, 128, 128, "half", 16, 0), ("bf16", 2, 14, 64, 32, "interleaved", 5, 1), ("f16", 3, 9, 96, 20, "half", 1, 0),
          ("f32", 1, 1, 32, 6, "interleaved", 7, 0), ("f16", 5, 5, 256, 256, "half", 16, 1), ("f32", 9, 18, 160, 96, "half", 8, 0), ("bf16", 4, 4, 224, 2, "half", 32, 0)]


@pytest.mark.parametrize("dtype,heads,q_heads,dim,rot,style,bs,layout", SHAPES)
def test_append_writes_the_formulas_bytes_and_nothing_else(dtype, heads, q_heads, dim, rot, style, bs, layout):
    s = Setup("e2m1", heads, dim, bs, [0, 37, 5, 0, 64], [1, 3, 0, 19, 130], layout=layout, seed=dim + heads)
    wide = rand(s, s.tokens, q_heads + 2 * heads, dim, dtype=KIND[dtype])                # q, k, v side by side
    q, k, v = wide[:, :q_heads], wide[:, q_heads:q_heads + heads], wide[:, q_heads + heads:]
    v[:, :, ::3] *= 2.0 ** -9                                                           # groups of unlike size
    pos = torch.randint(0, 500, (s.tokens,), device="cuda", generator=s.gen, dtype=torch.int32)
    table = table_of(rot, 500)
    q_out, before = torch.full_like(q, 7.0), s.pool.clone()
    s.cache.append(s.pool, 1, s.batch, q=q, k=k, v=v, q_out=q_out, rope=kvr.Rope(table, rot, style), positions=pos)
    s.ok()
    want_q = turn64(q, table, pos, rot, style)
    assert_within(q_out, want_q, U[dtype] * want_q.abs() + 2.0 ** -22 * 8)
    written = torch.cat([s.slots(r, c, t) for r, (c, t) in enumerate(zip(s.context, s.new))])
    # the turned k in fp32 as append rounds it, from an fp32 output
    turned = torch.zeros(s.tokens, heads, dim, device="cuda")
    s.cache.append(s.pool, 1, s.batch, q=k.float(), q_out=turned, rope=kvr.Rope(table, rot, style), positions=pos)
    for kv, x in ((0, turned), (1, v.float())):
        same_records(records(s, 1, kv)[written], pack(x), dim)
        x = x.double()
        got, scale = s.decode(1, kv)
        top = x.unflatten(-1, (-1, 16)).abs().amax(-1, keepdim=True)
        assert_within(got[written].unflatten(-1, (-1, 16)), x.unflatten(-1, (-1, 16)),
                      top / 6 * (1 + 2.0 ** -4) * (1 + 2.0 ** -10) + 7 * 2.0 ** -10 * scale[written][..., None, None])
    for layer in range(2):
        for kv in range(2):
            a, b = s.plane(layer, kv).clone(), s.plane(layer, kv, before).clone()
            if layer == 1:
                a[written] = 0
                b[written] = 0
            assert torch.equal(a, b)


def test_quantising_odd_values():
    """Zeros, the smallest and the largest numbers, ties, groups far below their head, and what is not finite."""
    s = Setup("e2m1", 4, 64, 16, [0], [9])
    x = torch.zeros(9, 4, 64, device="cuda")
    x[1] = 1e-40
    big = torch.finfo(torch.float32).max
    x[2, :, 3], x[2, :, 4] = big, -big
    x[3, 1, 5], x[3, 2, 6], x[3, 3, 31] = math.inf, -math.inf, math.nan
    x[3, 0] = 1.0
    x[4] = torch.linspace(-1, 1, 64, device="cuda")
    x[5, :, 7] = -1e-30
    # scale 1, group scale 448 and 1: the codes' ties, both signs
    x[6, :, 0] = 2688.0
    x[6, :, 16:32] = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -6], device="cuda")
    x[7, :, :16], x[7, :, 16:32], x[7, :, 32:48] = 2688.0, 6 * 2.0 ** -9, 6 * 2.0 ** -11       # subnormal group scale; none
    x[8] = -0.0
    s.cache.append(s.pool, 0, s.batch, k=x, v=x)
    out = torch.zeros(9, 4, 64, device="cuda")
    s.cache.read(s.pool, 0, s.batch, k=out)
    s.ok()
    same_records(records(s, 0, 0)[s.slots(0, 0, 9)], pack(x), 64)
    same_records(records(s, 0, 1)[s.slots(0, 0, 9)], pack(x), 64)
    assert (out[0] == 0).all() and (out[1] == 0).all() and torch.isfinite(out[2]).all()
    assert torch.isnan(out[3, 1:]).all() and (out[3, 0] == out[3, 0, 0]).all() and (out[3, 0, 0] - 1).abs() < 2.0 ** -20
    assert torch.equal(out[6, 0, 16:32].cpu(), torch.tensor([0, 1, 1, 2, 2, 4, 4, 6, -0., -1, -1, -2, -2, -4, -4, -6]))
    assert (out[7, :, 16:32] == 6 * 2.0 ** -9).all() and (out[7, :, 32:48] == 0).all()


@pytest.mark.parametrize("dtype,heads,dim,bs,layout", [("bf16", 8, 128, 16, 0), ("f16", 2, 64, 5, 1), ("f32", 3, 96, 1, 0), ("bf16", 1, 256, 8, 0), ("f32", 9, 32, 3, 1)])
def test_read_returns_what_the_cache_holds(dtype, heads, dim, bs, layout):
    s = Setup("e2m1", heads, dim, bs, [0, 7, 0, 33], [21, 40, 0, 1], layout=layout, seed=dim)
    k, v = s.fill(1)
    wide = torch.full((s.tokens, heads + 1, dim + 16), 5.0, dtype=KIND[dtype], device="cuda")
    k_out, v_out = wide[:, :heads, :dim], torch.zeros(heads, s.tokens, dim, dtype=KIND[dtype], device="cuda").transpose(0, 1)
    s.cache.read(s.pool, 1, s.batch, k=k_out, v=v_out)
    s.ok()
    for got, want in ((k_out, k), (v_out, v)):
        want = torch.cat([w[c:] for w, c in zip(want, s.context)])
        assert_within(got, want, (U[dtype] + 2.0 ** -24) * want.abs() + (2.0 ** -25 if dtype == "f16" else 0))
    assert (wide[:, heads] == 5).all() and (wide[..., dim:] == 5).all()


def test_read_of_any_bytes():
    """Codes, scales and groups' scales that append does not write."""
    s = Setup("e2m1", 3, 64, 4, [0], [300], seed=9)
    r = torch.randint(0, 256, (s.pool.numel(),), dtype=torch.uint8, device="cuda", generator=s.gen)
    s.pool.copy_(r)
    rec = s.pool.view(-1, 48)
    rec[:, 32:36] = (torch.rand(rec.shape[0], 1, device="cuda", generator=s.gen) * 4).view(torch.uint8)
    out = torch.zeros(300, 3, 64, device="cuda")
    s.cache.read(s.pool, 0, s.batch, v=out)
    want = s.decode(0, 1)[0][s.slots(0, 0, 300)]
    assert_within(out, want, 2.0 ** -24 * want.abs())


# ---- positions with several axes ---------------------------------------------------

def turned_by_axes(x, table, where, axes, rot, style, inverse=False):
    """The formula, pair by pair: each axis's pairs out of a turn by that axis's position."""
    out = x.double().clone()
    pair = torch.tensor(axes, device="cuda")
    for axis in range(max(axes) + 1):
        y = turn64(x, table, where[:, axis], rot, style, inverse)
        p = torch.nonzero(pair == axis)[:, 0]
        for c in ([p, p + rot // 2] if style == "half" else [2 * p, 2 * p + 1]):
            out[..., c] = y[..., c]
    return out


AXES = [("bf16", "bf16", 8, 32, 128, 128, "half", [16, 24, 24]), ("f16", "f16", 2, 6, 64, 64, "interleaved", [16, 16]), ("f32", "bf16", 1, 2, 80, 80, "half", [20, 20]),
        ("bf16", "e2m1", 2, 4, 128, 128, "half", "turns"), ("bf16", "e4m3", 2, 4, 96, 48, "interleaved", [5, 7, 12]), ("f32", "f16", 3, 3, 48, 22, "half", [3, 3, 3, 2]),
        ("f16", "int8", 2, 2, 256, 256, "interleaved", "turns"), ("f32", "f16", 1, 1, 64, 36, "interleaved", [9, 9]), ("bf16", "bf16", 2, 4, 256, 256, "half", [128])]


@pytest.mark.parametrize("dtype,fmt,heads,q_heads,dim,rot,style,parts", AXES)
def test_axes_turn_each_pair_by_its_own_position(dtype, fmt, heads, q_heads, dim, rot, style, parts):
    s = Setup(fmt, heads, dim, 16, [0, 9], [70, 33], seed=dim + rot)
    axes = [p % 3 for p in range(rot // 2)] if parts == "turns" else [i for i, n in enumerate(parts) for _ in range(n)]
    table, kind = table_of(rot, 300), KIND[dtype]
    where = torch.randint(0, 300, (s.tokens, max(axes) + 1), device="cuda", generator=s.gen, dtype=torch.int32)
    q, k, v = rand(s, s.tokens, q_heads, dim, dtype=kind), rand(s, s.tokens, heads, dim, dtype=kind), rand(s, s.tokens, heads, dim, dtype=kind)
    q_out, k_out = torch.zeros_like(q), torch.zeros(s.tokens, heads, dim, device="cuda")
    rope = kvr.Rope(table, rot, style, axes=axes)
    s.cache.append(s.pool, 0, s.batch, q=q, k=k, v=v, q_out=q_out, rope=rope, positions=where)
    s.cache.read(s.pool, 0, s.batch, k=k_out)
    s.ok()
    want = turned_by_axes(q, table, where, axes, rot, style)
    assert_within(q_out, want, U[dtype] * want.abs() + 2.0 ** -22 * 8)
    want = turned_by_axes(k, table, where, axes, rot, style)
    if fmt in ("bf16", "f16"):
        assert_within(k_out, want, U[fmt] * want.abs() + 2.0 ** -22 * 8)
    # the same bytes as one axis gives where all positions of a token are the same
    one, plain = torch.zeros_like(q), torch.zeros_like(q)
    same = where[:, :1].expand(-1, max(axes) + 1).contiguous()
    s.cache.append(s.pool, 0, s.batch, q=q, k=k, q_out=one, rope=rope, positions=same)
    by_axes = s.plane(0, 0).clone()
    s.cache.append(s.pool, 0, s.batch, q=q, k=k, q_out=plain, rope=kvr.Rope(table, rot, style), positions=where[:, 0].contiguous())
    assert torch.equal(one, plain) and torch.equal(by_axes, s.plane(0, 0))
    # and back
    back = torch.zeros(s.tokens, q_heads, dim, device="cuda")
    x = torch.zeros(s.tokens, q_heads, dim, device="cuda")
    s.cache.append(s.pool, 0, s.batch, q=q.float(), q_out=x, rope=rope, positions=where)
    s.cache.append(s.pool, 0, s.batch, q=x, q_out=back, rope=kvr.Rope(table, rot, style, inverse=True, axes=axes), positions=where)
    assert_within(back, q, 2.0 ** -20 * 8 + 0 * q.double())
    s.ok()


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_a_position_outside_the_table_leaves_its_token_out(axis):
    s = Setup("bf16", 2, 64, 16, [4], [5], seed=3)
    where = torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    where[2, axis] = -1 if axis == 1 else 50
    q, k = rand(s, 5, 2, 64), rand(s, 5, 2, 64)
    out, before = torch.full_like(q, 7.0), s.pool.clone()
    s.cache.append(s.pool, 0, s.batch, q=q, k=k, q_out=out, rope=kvr.Rope(table_of(64, 50), 64, axes=[0] * 10 + [1] * 10 + [2] * 12), positions=where)
    torch.cuda.synchronize()
    assert int(s.status) == kvr.DEV_BAD_POSITION and (out[2] == 7).all() and (out[[0, 1, 3, 4]] != 7).any()
    assert torch.equal(s.plane(0, 0)[s.slot(0, 6)], s.plane(0, 0, before)[s.slot(0, 6)])
    assert not torch.equal(s.plane(0, 0)[s.slot(0, 7)], s.plane(0, 0, before)[s.slot(0, 7)])


# ---- copies of blocks --------------------------------------------------------------

@pytest.mark.parametrize("fmt,heads,dim,bs,layers,layout", [("bf16", 8, 128, 16, 3, 0), ("e2m1", 2, 64, 5, 2, 1), ("e4m3", 3, 48, 1, 4, 0), ("f16", 1, 16, 7, 1, 1),
                                                            ("int8", 16, 256, 64, 2, 0), ("e2m1", 8, 128, 16, 5, 0)])
def test_copies_move_the_rows_asked_for(fmt, heads, dim, bs, layers, layout):
    nb = 60
    cache = kvr.Cache(layers, heads, dim, bs, nb, fmt, layout)
    gen = torch.Generator(device="cuda").manual_seed(bs)
    pool = torch.randint(0, 256, (cache.pool_bytes,), dtype=torch.uint8, device="cuda", generator=gen)
    ids = np.random.default_rng(bs).permutation(nb)
    pairs = [[int(ids[i]), int(ids[30 + i])] for i in range(20)]
    pairs += [[pairs[3][0], int(ids[52])], [-1, int(ids[53])], [-1, -5], [int(ids[54]), int(ids[54])]]       # shared source, places not in use, onto itself
    rows = [(i * 3) % (bs + 1) for i in range(len(pairs))]
    view = lambda p: (p.view(layers, 2, nb, bs, -1) if layout == 0 else p.view(nb, layers, 2, bs, -1).permute(1, 2, 0, 3, 4))     # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                                         # noqa: E731
    for n in (None, rows):
        want, got = pool.clone(), pool.clone()
        for i, (a, b) in enumerate(pairs):
            m = bs if n is None else n[i]
            if a >= 0:
                view(want)[:, :, b, :m] = view(pool)[:, :, a, :m]
        cache.copy(got, dev(pairs), rows=None if n is None else dev(n), status=status)
        torch.cuda.synchronize()
        assert int(status) == 0 and torch.equal(got, want)
    cache.copy(got, dev([[0, 0]])[:0], status=status)
    assert torch.equal(got, want)


def test_pairs_outside_the_pool_are_left_out_and_reported():
    cache = kvr.Cache(2, 2, 64, 16, 10, "bf16")
    pool = torch.randint(0, 256, (cache.pool_bytes,), dtype=torch.uint8, device="cuda")
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                                         # noqa: E731
    for bad, rows, code in (([10, 1], 16, kvr.DEV_BAD_BLOCK), ([1, 10], 16, kvr.DEV_BAD_BLOCK), ([1, -1], 16, kvr.DEV_BAD_BLOCK), ([-2, 1], 16, kvr.DEV_BAD_BLOCK),
                            ([2**31 - 1, 1], 16, kvr.DEV_BAD_BLOCK), ([2, 1], 17, kvr.DEV_BAD_LENGTH), ([2, 1], -1, kvr.DEV_BAD_LENGTH)):
        status, got, want = dev([0]), pool.clone(), pool.clone()
        cache.copy(got, dev([bad, [3, 4]]), rows=dev([rows, 16]), status=status)
        torch.cuda.synchronize()
        want.view(4, 10, -1)[:, 4] = want.view(4, 10, -1)[:, 3]
        assert int(status) == code and torch.equal(got, want)


def test_copies_in_a_captured_graph_follow_their_arrays():
    cache = kvr.Cache(2, 2, 64, 16, 40, "e2m1")
    pool = torch.randint(0, 256, (cache.pool_bytes,), dtype=torch.uint8, device="cuda")
    start = pool.clone()
    pairs = torch.full((6, 2), -1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.copy(pool, pairs)
    for now in ([[1, 2]], [[5, 6], [7, 8], [5, 9]], []):
        pairs.fill_(-1)
        if now:
            pairs[:len(now)] = torch.tensor(now, dtype=torch.int32)
        pool.copy_(start)
        graph.replay()
        want = start.clone().view(4, 40, -1)
        for a, b in now:
            want[:, b] = want[:, a]
        assert torch.equal(pool.view(4, 40, -1), want)


def test_copies_beyond_4_gib():
    cache = kvr.Cache(1, 8, 128, 16, 150_000, "bf16")                                # planes of 4.9 GB
    pool = torch.zeros(cache.pool_bytes, dtype=torch.uint8, device="cuda")
    tiles = pool.view(2, 150_000, -1)
    tiles[:, 149_998] = torch.randint(0, 256, tiles[:, 0].shape, dtype=torch.uint8, device="cuda")
    cache.copy(pool, torch.tensor([[149_998, 3], [149_998, 149_999]], dtype=torch.int32, device="cuda"))
    for b in (3, 149_999):
        assert torch.equal(tiles[:, b], tiles[:, 149_998])
    assert not tiles[:, 4].any() and not tiles[:, 149_997].any()


# ---- attend ------------------------------------------------------------------------

DIMS = [(8, 4, 128, 16), (2, 8, 128, 16), (1, 1, 64, 8), (3, 5, 96, 5), (4, 2, 256, 16), (12, 1, 64, 16), (5, 3, 32, 7), (8, 7, 64, 32), (1, 16, 192, 1), (17, 1, 128, 16),
        (2, 3, 224, 16), (1, 4, 160, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,group,dim,bs", DIMS)
def test_attend_single_tokens(dtype, heads, group, dim, bs):
    """One new token a request, contexts from none to thousands of tokens."""
    s = Setup("e2m1", heads, dim, bs, [0, 1, 14, 15, 16, 17, 63, 64, 255, 700, 3001], [1] * 11, seed=heads * dim)
    base.check_attend(s, heads * group, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,group,dim,bs", DIMS)
def test_attend_trees_with_empty_rows(dtype, heads, group, dim, bs):
    """Trees of up to 70 tokens (two mask words); rows that see nothing at all where there is no context."""
    s = Setup("e2m1", heads, dim, bs, [0, 0, 100, 511, 1000, 33, 0], [1, 7, 13, 64, 70, 0, 70], seed=heads * dim + 1, layout=heads % 2)
    mask, seen = base.tree(s, np.random.default_rng(dim), empty=0.15)
    out, lse, _ = base.check_attend(s, heads * group, dtype, mask, seen, strided=True)
    empty = torch.cat([~m.any(1) for m in seen])
    assert empty.any() and (out[empty] == 0).all() and (lse[empty] == -math.inf).all()


def test_attend_causal_chunks():
    s = Setup("e2m1", 2, 128, 16, [0, 300, 5], [200, 129, 1], seed=3)
    base.check_attend(s, 8, "bf16")


@pytest.mark.parametrize("new", [2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65])
def test_attend_every_tile_of_rows(new):
    s = Setup("e2m1", 2, 128, 16, [129, 40], [new, max(1, new // 2)], seed=new)
    mask, seen = base.tree(s, np.random.default_rng(new))
    base.check_attend(s, 8, "bf16", mask, seen)


@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("bs", [16, 5])
def test_attend_ignores_what_a_row_does_not_see(group, bs):
    """Some drafted tokens are NaN as append writes it (the head's scale), others hold the largest codes and scales there are, their groups' bytes
    too; rows that do not see them give the formula over what they see, rows that see a NaN give NaN."""
    s = Setup("e2m1", 2, 64, bs, [0, 50, 200], [9, 20, 33], seed=11)
    mask, seen = base.tree(s, np.random.default_rng(4))
    s.fill()
    for r, (c, t) in enumerate(zip(s.context, s.new)):
        one = kvr.Batch(torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([c + 1], dtype=torch.int32, device="cuda"),
                        s.arrays[2][r:r + 1].contiguous(), 1, c + t, s.status)
        x = torch.ones(1, 2, 64, device="cuda", dtype=torch.float32)
        x[0, 1, 5] = math.nan
        s.cache.append(s.pool, 0, one, k=x, v=x)
        s.plane(0, 1)[s.slot(r, c + 3)] = 0x7f                                       # any bytes: groups' scales of 480, a scale of 3e38
    finite = [torch.ones(t, dtype=torch.bool, device="cuda") for t in s.new]
    vals = [s.decode(0, i)[0] for i in (0, 1)]
    kv = [[x[s.slots(r, 0, c + t)] for r, (c, t) in enumerate(zip(s.context, s.new))] for x in vals]
    q = rand(s, s.tokens, 2 * group, 64)
    out, ws = torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    s.cache.attend(s.pool, 0, s.batch, q, out, ws, mask=mask)
    s.ok()
    at = 0
    for r, (c, t) in enumerate(zip(s.context, s.new)):
        clean = ~(seen[r][:, c + 1] | seen[r][:, c + 3])
        assert clean.any() and finite[r].all()
        for i in torch.nonzero(clean)[:, 0].tolist():
            keys = torch.nonzero(seen[r][i])[:, 0]
            for h in range(2 * group):
                kk, vv = kv[0][r][keys, h // group], kv[1][r][keys, h // group]
                p = torch.softmax(kk @ q[at + i, h].double() / 8.0, 0)
                assert_within(out[at + i, h], p @ vv, (U["f16"] + U["bf16"] + 2.0 ** -13) * (p @ vv.abs()) + 2.0 ** -12)
        hit = seen[r][:, c + 1]
        assert hit.any() and torch.isnan(out[at:at + t][hit][:, group:]).all()
        assert torch.isfinite(out[at:at + t][hit & ~seen[r][:, c + 3]][:, :group]).all()         # the other head of that token is finite
        at += t


@pytest.mark.parametrize("new", [1, 40])
def test_attend_large_and_unlike_values(new):
    """Scores far apart (the running maximum moves late and far), values of V across many magnitudes."""
    s = Setup("e2m1", 2, 128, 16, [900, 64], [new, new], seed=21, poison=False)
    s.fill()
    lens = [c + t for c, t in zip(s.context, s.new)]
    starts = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
    whole = kvr.Batch(starts, torch.zeros_like(s.arrays[1]), s.arrays[2], max(lens), max(lens), s.status)
    n = sum(lens)
    kk = rand(s, n, 2, 128, dtype=torch.float32) * torch.linspace(0.1, 3.0, n, device="cuda")[:, None, None]
    vv = rand(s, n, 2, 128, dtype=torch.float32) * torch.exp2(torch.randint(-6, 7, (n, 2, 1), device="cuda", generator=s.gen).float())
    s.cache.append(s.pool, 0, whole, k=kk, v=vv)
    vals = [s.decode(0, i)[0] for i in (0, 1)]
    base.check_attend(s, 8, "bf16", scale=0.5, kv=[[x[s.slots(r, 0, m)] for r, m in enumerate(lens)] for x in vals])


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("size", [1e-24, 1e-6, 1e6, 1e30])
def test_attend_small_and_large_values_of_v(size, new):
    s = Setup("e2m1", 2, 64, 16, [200], [new], seed=22)
    n = 200 + new
    whole = kvr.Batch(torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.zeros_like(s.arrays[1]), s.arrays[2], n, n, s.status)
    k, v = rand(s, n, 2, 64, dtype=torch.float32), rand(s, n, 2, 64, dtype=torch.float32)
    s.cache.append(s.pool, 0, whole, k=k, v=v * size)
    kv = [[s.decode(0, i)[0][s.slots(0, 0, n)]] for i in (0, 1)]
    q, ws = rand(s, new, 4, 64), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    out = torch.zeros(new, 4, 64, dtype=torch.bfloat16, device="cuda")
    s.cache.attend(s.pool, 0, s.batch, q, out, ws)
    s.ok()
    want, _, mag = base.attend64(s, q, *kv, 1 / 8.0, base.causal(s))
    assert_within(out, want, (U["f16"] + U["bf16"] + 2.0 ** -13) * mag + 2.0 ** -24 * 8 * size * 16)


@pytest.mark.parametrize("new,heads", [(1, 8), (33, 8), (1, 1), (3, 2)])
def test_attend_many_requests_and_many_pieces(new, heads):
    rng = np.random.default_rng(1)
    n = 600 if new == 1 else 40
    s = Setup("e2m1", heads, 64, 16, [int(x) for x in rng.integers(0, 40, n)], [new] * n, seed=31)
    base.check_attend(s, heads * 2, "bf16")
    s = Setup("e2m1", heads, 64, 16, [20000], [new], seed=32)
    base.check_attend(s, heads * 2, "bf16")
    if new > 1:
        s = Setup("e2m1", heads, 64, 16, [3, 5, 20000, 0], [0, new, new, 0], seed=33)
        mask, seen = base.tree(s, rng)
        base.check_attend(s, heads * 2, "bf16", mask, seen)


def test_attend_offsets_beyond_32_bits():
    """Blocks behind the first 4 GiB of a plane, from both ends of the pool."""
    heads, dim, bs = 8, 128, 16
    for new in (1, 20):
        s = Setup("e2m1", heads, dim, bs, [100, 30], [new, 1], layers=1, spare=(5 << 30) // (640 * bs), seed=41, poison=False)
        width = s.host_tables.shape[1]
        s.host_tables[:] = (s.nb - 1 - np.arange(2 * width).reshape(2, width)).astype(np.int32)
        s.arrays[2].copy_(torch.from_numpy(s.host_tables))
        n = 131 + new
        k, v = (rand(s, n, heads, dim) for _ in range(2))
        lens = [100 + new, 31]
        whole = kvr.Batch(torch.tensor([0, lens[0], n], dtype=torch.int32, device="cuda"), torch.zeros_like(s.arrays[1]), s.arrays[2], 120, 120, s.status)
        s.cache.append(s.pool, 0, whole, k=k, v=v)
        got = [torch.zeros(n, heads, dim, device="cuda") for _ in range(2)]
        s.cache.read(s.pool, 0, whole, k=got[0], v=got[1])
        assert got[0].abs().max() > 0.5
        base.check_attend(s, 32, "bf16", kv=[[x[:lens[0]].double(), x[lens[0]:].double()] for x in got])


def test_attend_leaves_out_what_does_not_fit():
    for new in (2, 20):
        s = Setup("e2m1", 2, 64, 16, [20, 20, 20], [new] * 3, seed=51)
        s.fill()
        q, ws = rand(s, 3 * new, 4, 64), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        for what in ("block", "tokens"):
            starts, context, tables = (x.clone() for x in s.arrays)
            if what == "block":
                tables[1, 1] = s.nb
            else:
                context[1] = 21
            out = torch.full_like(q, 3.0)
            s.status.zero_()
            s.cache.attend(s.pool, 0, kvr.Batch(starts, context, tables, new, 20 + new, s.status), q, out, ws)
            torch.cuda.synchronize()
            assert int(s.status) == (kvr.DEV_BAD_BLOCK if what == "block" else kvr.DEV_BAD_LENGTH)
            assert (out[:new] != 3).any() and (out[2 * new:] != 3).any() and (what == "block" or (out[new:2 * new] == 3).all())


# ---- together ----------------------------------------------------------------------

@pytest.mark.parametrize("new", [6, 40])
def test_a_step_on_another_stream_and_in_a_graph(new):
    """append (several axes) -> attend -> keep -> copy captured once and replayed with other lengths in the same arrays."""
    s = Setup("e2m1", 2, 64, 16, [100, 64], [new, new], layers=1, seed=71)
    s.fill()
    mask, _ = base.tree(s, np.random.default_rng(3))
    n = 2 * new
    q, kn, vn = rand(s, n, 8, 64), rand(s, n, 2, 64), rand(s, n, 2, 64)
    out, ws = torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    index, count = torch.tensor([[0, 2], [1, 5]], dtype=torch.int32, device="cuda"), torch.tensor([2, 2], dtype=torch.int32, device="cuda")
    where = torch.randint(0, 200, (n, 3), device="cuda", dtype=torch.int32)
    rope = kvr.Rope(table_of(64, 200), 64, axes=[0] * 8 + [1] * 12 + [2] * 12)
    b = kvr.Batch(*s.arrays, new, 100 + new, s.status)
    free = [x for x in range(s.nb) if x not in set(s.host_tables[:, :-(-(100 + new) // 16)].ravel().tolist())][:1]
    pairs = torch.tensor([[int(s.host_tables[0, 0]), free[0]]], dtype=torch.int32, device="cuda")

    def step():
        s.cache.append(s.pool, 0, b, q=q, k=kn, v=vn, q_out=q, rope=rope, positions=where)
        s.cache.attend(s.pool, 0, b, q, out, ws, mask=mask)
        s.cache.keep(s.pool, b, index, count)
        s.cache.copy(s.pool, pairs, status=s.status)

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


def test_a_4_bit_request_is_forked_suspended_compacted_and_answers_the_same():
    """The pool's movers and copies carry codes and scales: the answer after a fork, a suspend, a resume into other blocks and a compaction is the
    same, bit for bit, and the host holds 80 bytes a head."""
    c = kvr.Cache(2, 4, 128, 16, 200, "e2m1")
    pool = torch.zeros(c.pool_bytes, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, new = 500, 5
    with kvr.Pool(*c.geometry, 200, 64 << 20, initial_free_order=np.random.default_rng(1).permutation(200).astype(np.int32), device_pool=pool.data_ptr()) as p:
        st, blocks = p.admit(1, n)
        assert st == kvr.OK
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")       # noqa: E731
        k, v, q = (torch.randn(n, h, 128, device="cuda", generator=gen).bfloat16() for h in (4, 4, 8))
        for layer in range(2):
            c.append(pool, layer, kvr.Batch(i32([0, n]), i32([0]), i32(blocks)[None], n, n), k=k, v=v)
        ws = torch.zeros(c.workspace_bytes(), dtype=torch.uint8, device="cuda")

        def answer(rid):
            out = torch.zeros(2, new, 8, 128, dtype=torch.bfloat16, device="cuda")
            for layer in range(2):
                c.attend(pool, layer, kvr.Batch(i32([0, new]), i32([n - new]), i32(p.info(rid)[1]["blocks"])[None], new, n), q[:new], out[layer], ws)
            torch.cuda.synchronize()
            return out

        first = answer(1)
        assert p.fork(2, 1, n)[0] == kvr.OK and torch.equal(answer(2), first)
        assert p.suspend_to_host([1], kvr.SYNC)[0] == kvr.OK
        assert p.stats()["bytes_suspended"] == n * 2 * 2 * 4 * 80
        assert torch.equal(answer(2), first)
        assert p.resume_from_host([1], kvr.SYNC)[0] == kvr.OK and torch.equal(answer(1), first)
        assert p.info(1)[1]["blocks"].tolist() != blocks.tolist()
        assert len(p.compact()[1]) > 0 and torch.equal(answer(1), first) and torch.equal(answer(2), first)


@pytest.mark.parametrize("heads,group,dim,bs,new", [(2, 4, 128, 16, 1), (8, 4, 128, 8, 1), (2, 8, 64, 5, 2), (1, 1, 256, 16, 3), (2, 4, 128, 16, 20), (2, 8, 64, 5, 10)])
def test_a_call_that_gives_up_says_so_and_the_next_is_right(heads, group, dim, bs, new):
    """Both kernels' waits have limits: lowered on the host, on barriers that do complete later."""
    s = Setup("e2m1", heads, dim, bs, [900, 30, 0], [new] * 3, layers=1, seed=new)
    s.fill()
    mask, _ = base.tree(s, np.random.default_rng(new))
    q = rand(s, s.tokens, heads * group, dim)

    def attend():
        out, ws = torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        s.status.zero_()
        s.cache.attend(s.pool, 0, s.batch, q, out, ws, mask=mask)
        torch.cuda.synchronize()
        return out, int(s.status)

    want, status = attend()
    assert status == 0
    polls = kvr.lib().kvr_test_attend_polls
    for limit in (0, 1, 8, 100):
        was = polls(limit)
        try:
            out, status = attend()
        finally:
            polls(was)
        assert status == kvr.DEV_GAVE_UP if limit == 0 else status in (0, kvr.DEV_GAVE_UP)
        assert status or torch.equal(out, want)
        out, status = attend()
        assert status == 0 and torch.equal(out, want)


def test_two_calls_at_once_with_workspaces_of_their_own():
    """On two streams, several times; each answer is the one that the call gives alone."""
    a = Setup("e2m1", 8, 128, 16, [3000, 500, 70], [1, 1, 1], layers=1, seed=5)
    b = Setup("e2m1", 2, 64, 8, [4000, 9], [30, 7], layers=1, seed=6)
    both = []
    for s, heads in ((a, 32), (b, 8)):
        s.fill()
        q = rand(s, s.tokens, heads, s.dim)
        both.append((s, q, torch.zeros_like(q), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda"), torch.cuda.Stream()))
    want = []
    for s, q, out, ws, _ in both:
        s.cache.attend(s.pool, 0, s.batch, q, out, ws)
        torch.cuda.synchronize()
        want.append(out.clone())
        out.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, q, out, ws, stream in both:
            with torch.cuda.stream(stream):
                s.cache.attend(s.pool, 0, s.batch, q, out, ws)
    torch.cuda.synchronize()
    for (s, q, out, ws, _), x in zip(both, want):
        assert torch.equal(out, x)
        s.ok()


def test_rows_behind_the_last_request_stay_as_they_were():
    s = Setup("e2m1", 2, 128, 16, [40, 3], [1, 2], seed=8)
    s.fill()
    for grown in (1, 30):                        # the row kernel's tiles, and the tile kernel's
        new = s.batch if grown == 1 else kvr.Batch(*s.arrays, 30, 70, s.status)
        q = rand(s, 7, 8, 128)
        out, lse = torch.full_like(q, 5.0), torch.full((7, 8), 5.0, device="cuda")
        ws = torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        s.cache.attend(s.pool, 0, new, q, out, ws, lse=lse)
        s.ok()
        assert (out[3:] == 5).all() and (lse[3:] == 5).all() and (out[:3] != 5).any()


@pytest.mark.parametrize("heads,group,dim,bs,new", [(1, 4, 64, 8, 1), (1, 1, 64, 64, 1), (2, 4, 128, 128, 1), (8, 4, 128, 256, 1), (8, 2, 128, 48, 3), (20, 1, 128, 16, 1),
                                                    (7, 2, 256, 40, 2), (3, 4, 32, 9, 3), (4, 12, 96, 64, 4), (1, 16, 128, 2, 2)])
def test_attend_any_block_size_and_number_of_heads(heads, group, dim, bs, new):
    """Blocks that are smaller and larger than a stage of the loads, boxes of every size, groups of heads that do not divide; two layers, the second one read."""
    s = Setup("e2m1", heads, dim, bs, [1500, 0, 47, 400, 1], [new] * 5, seed=heads + dim + bs, layout=bs % 2)
    base.check_attend(s, heads * group, "bf16", layer=1)


@pytest.mark.parametrize("new", [1, 30])
def test_tables_cut_from_wider_ones(new):
    """Rows of a table that are views into wider ones, with ids behind them that are no blocks."""
    s = Setup("e2m1", 2, 128, 16, [100, 37], [new, new], seed=9)
    k, v = s.fill()
    q, ws = rand(s, s.tokens, 8, 128), torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    width = -(-(100 + new) // 16)
    wide = torch.full((2, 50), s.nb + 7, dtype=torch.int32, device="cuda")
    wide[:, 10:10 + width] = s.arrays[2][:, :width]
    out = [torch.zeros_like(q) for _ in range(2)]
    s.cache.attend(s.pool, 0, s.batch, q, out[0], ws)
    s.cache.attend(s.pool, 0, kvr.Batch(s.arrays[0], s.arrays[1], wide[:, 10:10 + width], new, 100 + new, s.status), q, out[1], ws)
    s.ok()
    assert torch.equal(*out)
