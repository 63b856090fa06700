"""What a row does not see has no influence on it, whatever lies there: rows that were never written, and scales of any size.

The bytes of some new tokens are replaced, and every row that does not see them has to come out as before, bit for bit: their
probability is zero, so no rounding of any other term may change.  Rows that do see them are held to the definition in 64
bits, within the bounds of test_gpu_cache.py.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_cache import KIND, U, Setup, assert_within, attend64, rand

pytestmark = pytest.mark.gpu

# heads, group, dim, block size, new tokens: one and two tiles of the row kernel, both shapes of the tile kernel with boxes of 16 and 8
# tokens and without, and the row kernel alone (256 channels)
SHAPES = [(2, 1, 64, 16, 7), (3, 2, 128, 16, 8), (2, 4, 128, 16, 20), (2, 8, 64, 8, 40), (4, 2, 128, 8, 70), (1, 3, 96, 7, 30), (1, 2, 256, 16, 40)]
CONTEXT = [0, 40, 127, 300]


class Trees:
    """Requests with trees of two branches below token 0: `odd` with every fourth token behind it, and all others."""

    def __init__(self, fmt, dtype, heads, group, dim, bs, new, seed, odd=1):
        self.s = s = Setup(fmt, heads, dim, bs, CONTEXT, [new] * len(CONTEXT), layers=1, seed=seed)
        self.q_heads, self.odd = heads * group, odd
        s.fill()
        i, j = np.ogrid[:new, :new]
        side = lambda x: (x == odd) | ((x > odd) & (x % 4 == 0))                     # noqa: E731
        rows = (j <= i) & ((j == 0) | (side(i) == side(j)))
        words = -(-new // 64)
        bits = np.zeros((s.tokens, words * 64), dtype=bool)
        self.seen = []
        for r, c in enumerate(CONTEXT):
            bits[s.starts[r]:s.starts[r] + new, :new] = rows
            m = torch.ones(new, c + new, dtype=torch.bool, device="cuda")
            m[:, c:] = torch.from_numpy(rows).cuda()
            self.seen.append(m)
        self.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int64)).cuda()
        self.q = rand(s, s.tokens, self.q_heads, dim, dtype=KIND[dtype])
        self.hit = torch.from_numpy(np.tile(rows[:, odd], len(CONTEXT))).cuda()      # [tokens]: rows that see `odd`
        assert self.hit.any() and not self.hit.all()

    def attend(self):
        s = self.s
        out, lse = torch.full_like(self.q, 9.0), torch.full((s.tokens, self.q_heads), 9.0, device="cuda")
        ws = torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
        s.cache.attend(s.pool, 0, s.batch, self.q, out, ws, lse=lse, mask=self.mask)
        s.ok()
        return out, lse

    def odd_rows(self, kv):
        """The bytes of token `odd` of every request, [requests, row bytes], to be assigned to."""
        s = self.s
        return s.plane(0, kv), torch.stack([s.slots(r, c + self.odd, 1)[0] for r, c in enumerate(CONTEXT)])

    def same_but_for_those_that_see_it(self, a, b):
        for x, y in zip(a, b):
            x, y = x[~self.hit], y[~self.hit]
            assert torch.isfinite(x).all() and torch.equal(x, y), "%d of %d rows changed" % (int((x != y).flatten(1).any(1).sum()), len(x))


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("heads,group,dim,bs,new", SHAPES)
def test_new_tokens_that_were_never_written(fmt, dtype, heads, group, dim, bs, new):
    """K, V and scales of a token left at 0xff (or V's codes alone): as bf16, f16, e4m3 and fp32 that is NaN."""
    t = Trees(fmt, dtype, heads, group, dim, bs, new, seed=new + dim)
    clean = t.attend()
    v, slots = t.odd_rows(1)
    v[slots, :heads * dim * (1 if fmt in ("e4m3", "int8") else 2)] = 0xff
    t.same_but_for_those_that_see_it(clean, t.attend())
    for kv in (0, 1):
        x, slots = t.odd_rows(kv)
        x[slots] = 0xff
    out, lse = t.attend()
    t.same_but_for_those_that_see_it(clean, (out, lse))
    assert torch.isnan(out[t.hit]).all()                      # (int8: by its scale)


@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("heads,group,dim,bs,new", SHAPES)
def test_a_single_nan_code_reaches_its_channel_in_rows_that_see_it(code, heads, group, dim, bs, new):
    t = Trees("e4m3", "bf16", heads, group, dim, bs, new, seed=new + dim + 1, odd=2)
    clean = t.attend()
    v, slots = t.odd_rows(1)
    channel, head = dim - 3, heads - 1
    v[slots, head * dim + channel] = code
    out, lse = t.attend()
    t.same_but_for_those_that_see_it(clean, (out, lse))
    assert torch.equal(lse, clean[1])
    nan = torch.isnan(out)
    want = torch.zeros_like(nan)
    want[t.hit.nonzero()[:, 0], head * group:, channel] = True
    assert torch.equal(nan, want)
    # the other channels of those rows are the formula's
    k64, v64 = ([x[t.s.slots(r, 0, c + new)] for r, c in enumerate(CONTEXT)] for x in (t.s.decode(0, 0)[0], torch.nan_to_num(t.s.decode(0, 1)[0])))
    ref, _, mag = attend64(t.s, t.q, k64, v64, 1 / math.sqrt(dim), t.seen)
    top = max(float(x.abs().max()) for x in v64)
    bound = (U["f16"] + U["bf16"] + 2.0 ** -13) * mag + 2.0 ** -24 * top * math.sqrt(CONTEXT[-1] + new)
    assert_within(torch.where(want, 0, out), torch.where(want, 0, ref), bound)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("size", [1e12, 1e30, -math.inf])
@pytest.mark.parametrize("heads,group,dim,bs,new", SHAPES)
def test_the_scale_of_a_token_that_a_row_does_not_see(fmt, size, heads, group, dim, bs, new):
    """V of one branch is far larger than all other: the other branch is as if it were not there, its own rows are right."""
    t = Trees(fmt, "bf16", heads, group, dim, bs, new, seed=new + dim + 2)
    s = t.s
    clean = t.attend()
    if math.isfinite(size):
        one = kvr.Batch(torch.arange(len(CONTEXT) + 1, dtype=torch.int32, device="cuda"), s.arrays[1] + t.odd, s.arrays[2], 1,
                        CONTEXT[-1] + new, s.status)
        s.cache.append(s.pool, 0, one, v=rand(s, len(CONTEXT), heads, dim, dtype=torch.float32) * size)
    else:                                                    # bytes that append does not write: a scale of infinity
        v, slots = t.odd_rows(1)
        if fmt == "bf16":
            v[slots] = torch.full((heads * dim,), size, dtype=torch.bfloat16, device="cuda").view(torch.uint8)
        else:
            v[slots, heads * dim:heads * dim + 4 * heads] = torch.full((heads,), -size, device="cuda").view(torch.uint8)
    out, lse = t.attend()
    t.same_but_for_those_that_see_it(clean, (out, lse))
    assert torch.equal(lse, clean[1])
    if not math.isfinite(size):
        assert not torch.isfinite(out[t.hit]).any()
        return
    kv = [[s.decode(0, i)[0][s.slots(r, 0, c + new)] for r, c in enumerate(CONTEXT)] for i in (0, 1)]
    want, _, mag = attend64(s, t.q, *kv, 1 / math.sqrt(dim), t.seen)
    u_p = U["bf16"] if fmt == "bf16" else U["f16"]
    # what a key adds is f16 against the largest |v| that the row sees
    top = torch.where(t.hit, max(float(x.abs().max()) for x in kv[1]), max(float(x[:c].abs().max()) if c else 0.0 for x, c in zip(kv[1], CONTEXT)))
    tiny = 0 if fmt == "bf16" else 2.0 ** -24 * math.sqrt(CONTEXT[-1] + new) * top[:, None, None]
    assert_within(out, want, (u_p + U["bf16"] + 2.0 ** -13) * mag + tiny + 2.0 ** -100)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,group,dim,bs,new", SHAPES)
def test_an_infinite_scale_beside_one_that_grows(fmt, heads, group, dim, bs, new):
    """An unseen scale of infinity must not keep the unit of a row from following a scale that the row does see."""
    t = Trees(fmt, "bf16", heads, group, dim, bs, new, seed=new + dim + 3)
    s = t.s
    one = kvr.Batch(torch.arange(len(CONTEXT) + 1, dtype=torch.int32, device="cuda"), s.arrays[1], s.arrays[2], 1, CONTEXT[-1] + new, s.status)
    s.cache.append(s.pool, 0, one, v=rand(s, len(CONTEXT), heads, dim, dtype=torch.float32) * 2.0 ** 24)      # token 0, which all see but `odd`
    clean = t.attend()
    v, slots = t.odd_rows(1)
    kv = [[s.decode(0, i)[0][s.slots(r, 0, c + new)] for r, c in enumerate(CONTEXT)] for i in (0, 1)]
    v[slots, heads * dim:heads * dim + 4 * heads] = torch.full((heads,), math.inf, device="cuda").view(torch.uint8)
    out, lse = t.attend()
    t.same_but_for_those_that_see_it(clean, (out, lse))
    want, _, mag = attend64(s, t.q, *kv, 1 / math.sqrt(dim), t.seen)
    top = max(float(x.abs().max()) for x in kv[1])
    bound = (U["f16"] + U["bf16"] + 2.0 ** -13) * mag + 2.0 ** -24 * top * math.sqrt(CONTEXT[-1] + new)
    assert_within(out[~t.hit], want[~t.hit], bound[~t.hit])
