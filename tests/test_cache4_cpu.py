"""The 4-bit cache, positions with several axes and copies of blocks without a GPU: geometry, and what the C entries and the binding refuse."""
import ctypes as C

import pytest
import torch

from paper_2608_30830_b200 import kvr
from test_cache_cpu import FAKE, batch, ref, rows, spec


def test_geometry_of_4_bit_caches():
    c = kvr.Cache(32, 8, 128, 16, 64, "e2m1")
    assert c.geometry == (32, 1, 8 * 80, 1, 16) and c.row_bytes == 640 and c.pool_bytes == 2 * 32 * 64 * 16 * 640
    assert kvr.bytes_per_token(*c.geometry[:4]) * 3.2 == kvr.bytes_per_token(32, 8, 128, 2)
    assert [kvr.Cache(1, 1, d, 4, 5, "e2m1").row_bytes for d in (32, 64, 96, 160, 192, 224, 256)] == [32, 48, 64, 96, 112, 144, 160]
    for d in (16, 48, 80, 112, 240):
        with pytest.raises(kvr.KvrError) as e:
            kvr.Cache(1, 1, d, 4, 5, "e2m1")
        assert e.value.status == kvr.ERR_GEOMETRY


def axes(n, of_pair):
    return kvr.RopeAxes(n, (C.c_uint8 * 128)(*of_pair))


def append_axes(rope=None, a=None, positions=FAKE, b=None):
    return kvr.lib().kvr_cache_append_axes(ref(spec()), FAKE, 0, ref(b or batch()), None, ref(rows()), None, None, ref(rope), ref(a), positions, None)


def test_append_axes_refuses():
    rope, good = kvr.RopeStruct(FAKE, 10, 64, 0, 0), axes(3, [0] * 16 + [1] * 8 + [2] * 8)
    for kw in (dict(a=None), dict(rope=None), dict(positions=None), dict(positions=FAKE + 2), dict(a=axes(0, [0] * 32)), dict(a=axes(5, [4] * 32)),
               dict(a=axes(2, [0] * 31 + [2])), dict(a=axes(-1, [0] * 32)), dict(rope=kvr.RopeStruct(FAKE, 10, 66, 0, 0))):
        assert append_axes(**{**dict(rope=rope, a=good), **kw}) == kvr.ERR_INVALID_ARG, kw
        assert kvr.last_error()
    empty = batch(n_tokens=0, n_req=0, token_start=None, context=None, tables=None)
    assert append_axes(rope=rope, a=good, b=empty) == kvr.OK
    assert append_axes(rope=rope, a=axes(3, [0] * 32 + [9] * 96), b=empty) == kvr.OK      # entries behind the pairs are not read


def test_copy_refuses():
    def copy(pairs=FAKE, rows=FAKE, n=3, status=None, pool=FAKE, s=None):
        return kvr.lib().kvr_cache_copy(ref(s or spec()), pool, pairs, rows, n, status, None)
    for kw in (dict(pool=None), dict(pool=FAKE + 8), dict(pairs=None), dict(pairs=FAKE + 4), dict(rows=FAKE + 2), dict(status=FAKE + 1), dict(n=-1), dict(n=2**31 - 1)):
        assert copy(**kw) == kvr.ERR_INVALID_ARG, kw
    assert copy(s=spec(head_dim=65)) == kvr.ERR_GEOMETRY
    assert copy(pairs=None, rows=None, n=0) == kvr.OK


def test_the_binding_refuses_malformed_tensors(monkeypatch):
    monkeypatch.setattr(kvr, "_device", lambda: (kvr._torch or kvr._use_torch()) and -1)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)                    # noqa: E731
    table = torch.zeros(10, 32, 2)
    for bad in ([0] * 31, [0] * 31 + [4], [-1] + [0] * 31, []):
        with pytest.raises(ValueError):
            kvr.Rope(table, 64, axes=bad)
    assert kvr.Rope(table, 64, axes=[0] * 16 + [2] * 16).axes.axes == 3
    c = kvr.Cache(1, 2, 64, 16, 8, "e2m1")
    pool, b = torch.zeros(c.pool_bytes, dtype=torch.uint8), kvr.Batch(i32(3), i32(2), i32(2, 4), 1, 10)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    for where in (None, i32(2), i32(2, 2), i32(3, 3), i32(2, 3).long(), i32(3, 2).t()):
        with pytest.raises(ValueError):
            c.append(pool, 0, b, k=k, rope=kvr.Rope(table, 64, axes=[0] * 16 + [2] * 16), positions=where, stream=0)
    with pytest.raises(ValueError):                                        # several axes' positions for a table of one
        c.append(pool, 0, b, k=k, rope=kvr.Rope(table, 64), positions=i32(2, 3), stream=0)
    for pairs, n in ((i32(3), None), (i32(3, 3), None), (i32(3, 2).long(), None), (i32(2, 3).t(), None), (i32(3, 2), i32(2)), (i32(3, 2), i32(3).long()), (i32(3, 2), i32(3, 1))):
        with pytest.raises(ValueError):
            c.copy(pool, pairs, rows=n, stream=0)
    with pytest.raises(ValueError):
        c.copy(pool[:-1], i32(3, 2), stream=0)
    with pytest.raises(ValueError):
        c.copy(pool, i32(3, 2), status=torch.zeros(1), stream=0)
