"""How attention shares a call out (heads of a CTA, pieces of a segment, openings), and the rounding of codes."""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_gpu_cache import Setup, check_attend, rand, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("heads,group,new", [(1, 4, 1), (3, 8, 2), (5, 2, 1), (7, 3, 5), (8, 8, 2), (12, 4, 1), (12, 1, 16),
                                             (8, 6, 3), (3, 16, 9)])
def test_few_requests_of_many_heads(fmt, dtype, heads, group, new):
    """One to three requests, cut into as many pieces as the GPU has SMs; heads that do not divide among the CTAs."""
    for context in ([3000], [0, 2049], [700, 1, 1500]):
        s = Setup(fmt, heads, 128, 16, context, [new] * len(context), seed=heads + group)
        mask, seen = tree(s, np.random.default_rng(new))
        check_attend(s, heads * group, dtype, mask, seen)


@pytest.mark.parametrize("heads,new", [(8, 1), (3, 2)])
def test_bounds_far_above_the_lengths(heads, new):
    """max_tokens and max_new change how a call is shared out, not what it answers."""
    s = Setup("int8", heads, 128, 16, [900, 40], [new, new], seed=7)
    s.batch.struct.max_tokens = 1 << 22
    check_attend(s, heads * 4, "bf16")
    s.batch.struct.max_new = 60
    check_attend(s, heads * 4, "bf16")


def test_more_units_than_are_numbered_is_refused():
    s = Setup("bf16", 8, 128, 16, [100], [1], seed=8)
    q, out = rand(s, 1, 32, 128), torch.full((1, 32, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(s.cache.workspace_bytes(), dtype=torch.uint8, device="cuda")
    s.batch.struct.max_tokens, s.batch.struct.max_new = 1 << 30, 1 << 20
    with pytest.raises(kvr.KvrError):
        s.cache.attend(s.pool, 0, s.batch, q, out, ws)
    torch.cuda.synchronize()
    assert (out == 9).all() and not ws.any()


@pytest.mark.parametrize("fmt,largest", [("e4m3", 448.0), ("int8", 127.0)])
@pytest.mark.parametrize("exponent", [-125, -101, -99, -60, 0, 60, 110])
def test_codes_are_those_of_the_divided_value(fmt, largest, exponent):
    """round(x / scale) with the quotient rounded to fp32 once, over the whole range of magnitudes; signed zeros too."""
    n, dim, bs = 64, 128, 16
    cache = kvr.Cache(1, 1, dim, bs, n // bs, fmt)
    pool = torch.zeros(cache.pool_bytes, dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")           # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(exponent + 200)
    # a magnitude of its own for each token, elements down to far below it; some lie half way between two codes
    x = torch.randn(n, 1, dim, generator=gen, device="cuda") * torch.exp2(torch.randint(-12, 1, (n, 1, dim), generator=gen, device="cuda").float())
    x[:, :, 1] = x.abs().amax(-1) * 1.5
    x[:, :, 2:64] = torch.round(x[:, :, 2:64] * 8) * x[:, :, 1:2] / 127 * 0.5
    x[:, :, 5], x[:, :, 6] = 0.0, -0.0
    x = torch.ldexp(x, i32(exponent))
    cache.append(pool, 0, kvr.Batch(i32([0, n]), i32([0]), i32([list(range(n // bs))]), n, n), k=x)
    rows = pool[:n * cache.row_bytes].view(n, cache.row_bytes)
    scale = rows[:, dim:dim + 4].contiguous().view(torch.float32)
    want = (x[:, 0].abs().amax(-1, keepdim=True) * float(np.float32(1) / np.float32(largest))).clamp_min(2.0 ** -126)
    assert torch.equal(scale, want)
    quotient = torch.from_numpy(x[:, 0].cpu().numpy() / scale.cpu().numpy())
    if fmt == "int8":
        codes = quotient.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    else:
        codes = quotient.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(rows[:, :dim].cpu(), codes)


@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
def test_turns_round_each_product_and_each_sum(style, inverse):
    """a cos - b sin with three roundings, whatever a compiler would contract: equal bits to separate fp32 operations."""
    n, heads, dim, rot = 50, 3, 128, 96
    cache = kvr.Cache(1, heads, dim, 16, 4, "bf16")
    pool = torch.zeros(cache.pool_bytes, dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")           # noqa: E731
    table = torch.empty(n, rot // 2, 2, device="cuda")
    kvr.rope_table(table)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(n, heads, dim, generator=gen, device="cuda")
    out = torch.zeros_like(q)
    cache.append(pool, 0, kvr.Batch(i32([0, n]), i32([0]), i32([[0, 1, 2, 3]]), n, n), q=q, q_out=out, rope=kvr.Rope(table, rot, style, inverse))
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if style == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    cos, sin = table[:, None, :, 0], table[:, None, :, 1] * (-1 if inverse else 1)
    want = q.clone()
    want[..., first] = q[..., first] * cos - q[..., second] * sin
    want[..., second] = q[..., second] * cos + q[..., first] * sin
    assert torch.equal(out, want)
