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
