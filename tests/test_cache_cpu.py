"""The operators over the paged cache without a GPU: geometry, rotary frequencies against their formulas, and what the
C entries and the binding refuse before anything is launched."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr

FAKE = 1 << 20                                    # a pointer that no call here may follow


def test_geometry_of_each_format():
    assert kvr.Cache(32, 8, 128, 16, 64, "bf16").geometry == (32, 8, 128, 2, 16)
    assert kvr.Cache(32, 8, 128, 16, 64, "f16").geometry == (32, 8, 128, 2, 16)
    for fmt in ("e4m3", "int8"):
        c = kvr.Cache(32, 8, 128, 16, 64, fmt)
        assert c.geometry == (32, 1, 8 * 128 + 32, 1, 16) and c.row_bytes == 1056
        assert kvr.bytes_per_token(*c.geometry[:4]) == 2 * 32 * 1056
        assert kvr.Cache(2, 3, 80, 4, 5, fmt).row_bytes == 240 + 16        # 12 bytes of scales, padded
        assert kvr.Cache(2, 5, 16, 4, 5, fmt).row_bytes == 80 + 32
    assert kvr.Cache(2, 3, 80, 4, 5, "bf16").pool_bytes == 2 * 2 * 5 * 4 * 480


@pytest.mark.parametrize("bad", [dict(layers=0), dict(kv_heads=0), dict(head_dim=8), dict(head_dim=72), dict(head_dim=272),
                                 dict(block_size=0), dict(num_blocks=0), dict(fmt=7), dict(fmt=-1), dict(layout=2),
                                 dict(kv_heads=1 << 16, head_dim=256, block_size=64)])
def test_bad_caches_are_refused(bad):
    args = dict(layers=1, kv_heads=2, head_dim=64, block_size=16, num_blocks=4, fmt="bf16", layout=0)
    args.update(bad)
    with pytest.raises(kvr.KvrError) as e:
        kvr.Cache(**args)
    assert e.value.status in (kvr.ERR_GEOMETRY, kvr.ERR_INVALID_ARG)
    spec = kvr.CacheSpec(args["layers"], args["kv_heads"], args["head_dim"], args["block_size"], args["num_blocks"],
                         {"bf16": 0}.get(args["fmt"], args["fmt"]), args["layout"])
    assert kvr.lib().kvr_attend_workspace(C.byref(spec)) == 0


def test_null_geometry():
    g = kvr.Geometry()
    assert kvr.lib().kvr_cache_geometry(None, C.byref(g)) == kvr.ERR_INVALID_ARG
    assert kvr.lib().kvr_cache_geometry(C.byref(kvr.CacheSpec(1, 1, 64, 16, 1, 0, 0)), None) == kvr.ERR_INVALID_ARG


# ---- frequencies: the formulas of include/kvr.h, in numpy -------------------------------

def test_plain_linear_and_base_frequencies():
    p = np.arange(32)
    f, m = kvr.rope_frequencies(64, base=10000.0)
    assert m == 1.0 and np.allclose(f, 10000.0 ** (-2 * p / 64), rtol=1e-14)
    f, m = kvr.rope_frequencies(64, base=10000.0, kind=kvr.SCALE_LINEAR, factor=4.0)
    assert m == 1.0 and np.allclose(f, 10000.0 ** (-2 * p / 64) / 4, rtol=1e-14)
    f, m = kvr.rope_frequencies(64, base=10000.0, kind=kvr.SCALE_BASE, factor=4.0)
    assert m == 1.0 and np.allclose(f, (10000.0 * 4.0 ** (64 / 62)) ** (-2 * p / 64), rtol=1e-13)
    # the slowest pair is slowed by the factor itself
    assert np.isclose(f[-1], 10000.0 ** (-62 / 64) / 4, rtol=1e-12) and f[0] == 1.0


def test_banded_frequencies():
    n, base, s, lo, hi, orig = 128, 500000.0, 8.0, 1.0, 4.0, 8192
    theta = base ** (-2 * np.arange(n // 2) / n)
    w = 2 * math.pi / theta
    t = np.clip((orig / w - lo) / (hi - lo), 0, 1)
    f, m = kvr.rope_frequencies(n, base=base, kind=kvr.SCALE_BANDS, factor=s, low=lo, high=hi, original=orig)
    assert m == 1.0 and np.allclose(f, theta * (t + (1 - t) / s), rtol=1e-13)
    assert np.array_equal(f[w < orig / hi], kvr.rope_frequencies(n, base=base)[0][w < orig / hi])
    assert np.allclose(f[w > orig / lo], theta[w > orig / lo] / s, rtol=1e-13)
    assert 0 < ((w >= orig / hi) & (w <= orig / lo)).sum() < n // 2


def test_ramped_frequencies():
    n, base, s, lo, hi, orig = 128, 10000.0, 16.0, 1.0, 32.0, 4096
    p = np.arange(n // 2)
    theta = base ** (-2 * p / n)
    at = lambda x: n * math.log(orig / (2 * math.pi * x)) / (2 * math.log(base))   # noqa: E731
    a, b = max(math.floor(at(hi)), 0), min(math.ceil(at(lo)), n - 1)
    t = 1 - np.clip((p - a) / (b - a), 0, 1)
    f, m = kvr.rope_frequencies(n, base=base, kind=kvr.SCALE_RAMP, factor=s, low=lo, high=hi, original=orig)
    assert np.allclose(f, theta * (t + (1 - t) / s), rtol=1e-13) and np.isclose(m, 0.1 * math.log(s) + 1, rtol=1e-14)
    assert 0 < a < b < n // 2
    assert kvr.rope_frequencies(n, base=base, kind=kvr.SCALE_RAMP, factor=1.0, low=lo, high=hi, original=orig)[1] == 1.0


@pytest.mark.parametrize("bad", [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=258), dict(base=1.0), dict(base=math.nan), dict(base=math.inf),
                                 dict(kind=5), dict(kind=-1), dict(kind=kvr.SCALE_LINEAR, factor=0.5), dict(kind=kvr.SCALE_LINEAR, factor=math.nan),
                                 dict(kind=kvr.SCALE_BASE, rot_dim=2, factor=2.0), dict(kind=kvr.SCALE_BANDS, factor=2.0, original=0),
                                 dict(kind=kvr.SCALE_BANDS, factor=2.0, original=10, low=4.0, high=4.0), dict(kind=kvr.SCALE_RAMP, factor=2.0, original=10, low=0.0)])
def test_bad_scalings_are_refused(bad):
    args = dict(rot_dim=64)
    args.update(bad)
    with pytest.raises(kvr.KvrError) as e:
        kvr.rope_frequencies(**args)
    assert e.value.status == kvr.ERR_INVALID_ARG


# ---- refusals of the C entries ------------------------------------------------------------

SPEC = (1, 2, 64, 16, 8, kvr.CACHE_BF16, 0)


def spec(**kw):
    s = kvr.CacheSpec(*SPEC)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def batch(**kw):
    b = kvr.BatchStruct(2, 3, 2, 40, 4, FAKE, FAKE, FAKE, None)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def rows(heads=2, **kw):
    r = kvr.Rows(FAKE, heads * 64, 64, heads, kvr.BF16)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def ref(x):
    return None if x is None else C.byref(x)


BAD_BATCHES = [None, dict(n_req=-1), dict(n_tokens=-1), dict(max_new=-1), dict(max_tokens=-1), dict(table_stride=-1), dict(n_req=0),
               dict(token_start=None), dict(context=None), dict(tables=None), dict(table_stride=0), dict(token_start=FAKE + 2), dict(status=FAKE + 1)]
BAD_ROWS = [dict(data=None), dict(data=FAKE + 8), dict(type=3), dict(type=-1), dict(heads=0), dict(token_stride=129), dict(head_stride=-64),
            dict(token_stride=1 << 50)]


def append(s=SPEC, b=None, q=None, k=None, v=None, q_out=None, rope=None, positions=None, pool=FAKE, layer=0):
    return kvr.lib().kvr_cache_append(ref(s if isinstance(s, kvr.CacheSpec) else spec()), pool, layer, ref(b), ref(q), ref(k), ref(v), ref(q_out),
                                      ref(rope), positions, None)


def attend(b=None, q=None, out=None, lse=FAKE, mask=None, words=0, scale=1.0, ws=FAKE, ws_bytes=None, pool=FAKE, layer=0, s=None):
    s = s or spec()
    return kvr.lib().kvr_cache_attend(ref(s), pool, layer, ref(b), ref(q), ref(out), lse, mask, words, scale, ws,
                                      kvr.lib().kvr_attend_workspace(ref(s)) if ws_bytes is None else ws_bytes, None)


def test_append_refuses():
    bad = kvr.ERR_INVALID_ARG
    good = dict(b=batch(), q=rows(4), k=rows(), v=rows(), q_out=rows(4))
    rope = lambda *a: kvr.RopeStruct(*a)                                   # noqa: E731
    for change in [dict(pool=None), dict(pool=FAKE + 8), dict(layer=-1), dict(layer=1), dict(q_out=None), dict(q=None), dict(k=rows(3)), dict(v=rows(4)),
                   dict(k=rows(type=kvr.F16)), dict(v=rows(type=kvr.F32)), dict(q_out=rows(2)), dict(q_out=rows(4, type=kvr.F16)),
                   dict(q_out=rows(4, token_stride=0)), dict(q_out=rows(4, head_stride=0)), dict(q=None, k=None, v=None, q_out=None),
                   dict(positions=FAKE + 2), dict(rope=rope(None, 10, 64, 0, 0)), dict(rope=rope(FAKE + 8, 10, 64, 0, 0)), dict(rope=rope(FAKE, 0, 64, 0, 0)),
                   dict(rope=rope(FAKE, 10, 66, 0, 0)), dict(rope=rope(FAKE, 10, 0, 0, 0)), dict(rope=rope(FAKE, 10, 31, 0, 0)), dict(rope=rope(FAKE, 10, 64, 2, 0))] + \
                  [dict(b=None if c is None else batch(**c)) for c in BAD_BATCHES] + [dict(k=rows(**c)) for c in BAD_ROWS]:
        assert append(**{**good, **change}) == bad, change
        assert kvr.last_error()
    assert append(s=spec(head_dim=65), **good) == kvr.ERR_GEOMETRY
    # nothing to do: no launch, so no CUDA either
    assert append(**{**good, "b": batch(n_tokens=0, n_req=0, token_start=None, context=None, tables=None)}) == kvr.OK


def test_read_refuses():
    def read(b=None, k=None, v=None, pool=FAKE, layer=0):
        return kvr.lib().kvr_cache_read(ref(spec()), pool, layer, ref(b), ref(k), ref(v), None)
    good = dict(b=batch(), k=rows(), v=rows())
    for change in [dict(pool=None), dict(layer=1), dict(k=None, v=None), dict(k=rows(3)), dict(k=rows(type=kvr.F16)), dict(k=rows(token_stride=0)),
                   dict(v=rows(head_stride=32))] + [dict(b=None if c is None else batch(**c)) for c in BAD_BATCHES] + [dict(v=rows(**c)) for c in BAD_ROWS]:
        assert read(**{**good, **change}) == kvr.ERR_INVALID_ARG, change
    assert read(b=batch(n_tokens=0), k=rows()) == kvr.OK


def test_attend_refuses():
    good = dict(b=batch(), q=rows(4), out=rows(4))
    for change in [dict(pool=None), dict(layer=2), dict(q=None), dict(out=None), dict(out=rows(2)), dict(q=rows(4, type=kvr.F16), out=rows(4, type=kvr.F16)),
                   dict(q=rows(4, type=kvr.F32), out=rows(4, type=kvr.F32)), dict(out=rows(4, type=kvr.F16)), dict(q=rows(3), out=rows(3)),
                   dict(out=rows(4, head_stride=0)), dict(scale=math.inf), dict(scale=math.nan), dict(mask=FAKE, words=0), dict(mask=FAKE + 4, words=1),
                   dict(mask=FAKE, words=1, b=batch(max_new=65)), dict(lse=FAKE + 2), dict(ws=None), dict(ws=FAKE + 128), dict(ws_bytes=1000)] + \
                  [dict(b=None if c is None else batch(**c)) for c in BAD_BATCHES] + [dict(q=rows(4, **{k: v for k, v in c.items() if k != "heads"}))
                                                                                     for c in BAD_ROWS if "heads" not in c]:
        assert attend(**{**good, **change}) == kvr.ERR_INVALID_ARG, change
    f16 = spec(format=kvr.CACHE_F16)
    assert attend(s=f16, **good) == kvr.ERR_INVALID_ARG                  # bf16 queries over an f16 cache
    assert attend(**{**good, "b": batch(n_tokens=0)}) == kvr.OK


def test_keep_refuses():
    def keep(b=None, index=FAKE, stride=4, count=FAKE, pool=FAKE):
        return kvr.lib().kvr_cache_keep(ref(spec()), pool, ref(b), index, stride, count, None)
    for change in [dict(pool=None), dict(index=None), dict(count=None), dict(stride=-1), dict(stride=0), dict(index=FAKE + 2), dict(count=FAKE + 1),
                   dict(b=batch(n_req=70000))] + [dict(b=None if c is None else batch(**c)) for c in BAD_BATCHES]:
        assert keep(**{"b": batch(), **change}) == kvr.ERR_INVALID_ARG, change
    assert keep(b=batch(n_tokens=0)) == kvr.OK


def test_binding_refuses_malformed_tensors(monkeypatch):
    """Shapes, types and strides are checked before a pointer is taken.  Host tensors stand in for device tensors here:
    their device ordinal is -1."""
    monkeypatch.setattr(kvr, "_device", lambda: (kvr._torch or kvr._use_torch()) and -1)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)                    # noqa: E731
    kvr.Batch(i32(3), i32(2), i32(2, 4), 1, 10)
    for args in [(i32(2), i32(2), i32(2, 4)), (i32(3), i32(2), i32(3, 4)), (i32(3).long(), i32(2), i32(2, 4)), (i32(3), i32(2), i32(2, 4).long()),
                 (i32(3), i32(2), i32(4, 2).t()), (i32(3), i32(2), i32(1, 4).expand(2, 4)), (i32(6)[::2], i32(2), i32(2, 4))]:
        with pytest.raises(ValueError):
            kvr.Batch(*args, 1, 10)
    assert kvr.Batch(i32(3), i32(2), i32(2, 8)[:, :4], 1, 10).struct.table_stride == 8
    with pytest.raises(ValueError):
        kvr.Rope(torch.zeros(10, 16, 2), 64)
    with pytest.raises(ValueError):
        kvr.Rope(torch.zeros(10, 32, 2, dtype=torch.float64), 64)
    with pytest.raises(KeyError):
        kvr.Rope(torch.zeros(10, 32, 2), 64, "other")
    c = kvr.Cache(1, 2, 64, 16, 8)
    b = kvr.Batch(i32(3), i32(2), i32(2, 4), 1, 10)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)                  # noqa: E731
    pool, ws = torch.zeros(c.pool_bytes, dtype=torch.uint8), torch.zeros(16, dtype=torch.uint8)
    for q, out in [(bf(2, 4, 32), bf(2, 4, 32)), (bf(2, 4, 128)[..., ::2], bf(2, 4, 64)), (bf(2, 4, 64), bf(3, 4, 64)), (bf(2, 4, 64).double(), bf(2, 4, 64))]:
        with pytest.raises(ValueError):
            c.attend(pool, 0, b, q, out, ws)
    for kw in [dict(lse=torch.zeros(2, 2)), dict(lse=torch.zeros(2, 4).double()), dict(mask=torch.zeros(1, 1, dtype=torch.int64)),
               dict(mask=torch.zeros(2, 1, dtype=torch.int32))]:
        with pytest.raises(ValueError):
            c.attend(pool, 0, b, bf(2, 4, 64), bf(2, 4, 64), ws, **kw)
    with pytest.raises(ValueError):
        c.attend(pool[:-1], 0, b, bf(2, 4, 64), bf(2, 4, 64), ws)
    with pytest.raises(ValueError):
        c.append(pool, 0, b, k=bf(2, 2, 64), v=bf(3, 2, 64))
    with pytest.raises(ValueError):
        c.append(pool, 0, b, k=bf(2, 2, 64), v=bf(2, 2, 64), positions=i32(3))
    with pytest.raises(ValueError):
        c.keep(pool, b, i32(3, 2), i32(2))
    with pytest.raises(kvr.KvrError):                                       # what the binding lets pass the library checks
        c.attend(pool, 5, b, bf(2, 4, 64), bf(2, 4, 64), ws, stream=0)
