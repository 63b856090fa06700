"""What the binding of the cache operators refuses, and what it hands to the library, without a GPU.

Host tensors stand in for device tensors (their device ordinal is -1), and a recorder stands in for the library, so that
nothing is launched whatever is let pass.
"""
import pytest
import torch

from paper_2608_30830_b200 import kvr


class Recorder:
    """Takes the place of the loaded library: keeps a copy of each call's kvr_batch and returns KVR_OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, [a._obj for a in args if hasattr(a, "_obj")], args))
            return kvr.OK
        return entry

    def batch(self):
        return next(x for x in self.calls[-1][1] if isinstance(x, kvr.BatchStruct))


@pytest.fixture
def library(monkeypatch):
    kvr.lib()
    kvr._use_torch()
    monkeypatch.setattr(kvr, "_device", lambda: -1)
    cache = kvr.Cache(1, 2, 64, 16, 8)                        # made by the library itself
    recorder = Recorder()
    monkeypatch.setattr(kvr, "_lib", recorder)
    recorder.cache = cache
    recorder.pool = torch.zeros(cache.pool_bytes, dtype=torch.uint8)
    return recorder


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def test_a_rotary_table_is_written_only_into_its_own_shape(library):
    kvr.rope_table(torch.zeros(10, 32, 2), stream=0)
    assert library.calls[-1][0] == "kvr_rope_table" and library.calls[-1][2][1:4] == (64, 0, 10)
    made = len(library.calls)
    for shape in [(10, 32, 1), (10, 32, 0), (10, 32, 3), (10, 64), (10, 32, 2, 1)]:
        with pytest.raises(ValueError):
            kvr.rope_table(torch.zeros(shape), stream=0)
    assert len(library.calls) == made


@pytest.mark.parametrize("width,bound", [(3, 48), (8, 100)])
def test_tables_cut_from_wider_ones_end_with_their_rows(library, width, bound):
    """Rows are `stride` entries apart, but only `width` of them are the table's: no request may reach into what follows (which
    for the last row lies beyond the memory)."""
    wide = i32(2, 8)
    b = kvr.Batch(i32(3), i32(2), wide[:, 8 - width:], 4, 100)
    assert b.struct.table_stride == 8
    c, pool = library.cache, library.pool
    c.append(pool, 0, b, k=bf(2, 2, 64), stream=0)
    assert library.batch().max_tokens == bound
    c.read(pool, 0, b, k=bf(2, 2, 64), stream=0)
    assert library.batch().max_tokens == bound
    c.attend(pool, 0, b, bf(2, 4, 64), bf(2, 4, 64), i32(4), stream=0)
    assert library.batch().max_tokens == bound
    c.keep(pool, b, i32(2, 1), i32(2), stream=0)
    assert library.batch().max_tokens == bound
    b.struct.max_tokens = 20                                  # a bound that is lower stays
    c.read(pool, 0, b, k=bf(2, 2, 64), stream=0)
    assert library.batch().max_tokens == 20


def test_calls_over_one_batch_do_not_share_their_struct(library):
    """A call of another thread may come while the library still reads this one's (it is called without the interpreter's lock)."""
    b = kvr.Batch(i32(3), i32(2), i32(2, 8), 4, 100)
    c, pool = library.cache, library.pool
    c.append(pool, 0, b, k=bf(5, 2, 64), stream=0)
    first = library.batch()
    c.keep(pool, b, i32(2, 1), i32(2), stream=0)
    c.read(pool, 0, b, k=bf(7, 2, 64), stream=0)
    assert first.n_tokens == 5 and library.batch().n_tokens == 7 and library.batch() is not first
    assert b.struct.n_tokens == 0


def test_keep_does_not_guess_where_the_rows_end(library):
    """token_start need not begin at 0: a part of a step's requests has its rows further on."""
    c, pool = library.cache, library.pool
    b = kvr.Batch(torch.tensor([100, 104, 108], dtype=torch.int32), i32(2), i32(2, 8), 4, 100)
    c.keep(pool, b, i32(2, 1), i32(2), stream=0)
    assert library.batch().n_tokens >= 108
    c.keep(pool, kvr.Batch(i32(1), i32(0), i32(0, 8), 4, 100), i32(0, 1), i32(0), stream=0)
    assert library.batch().n_tokens == 0                      # no requests: no tokens either


def test_calls_without_any_tensor_are_refused_as_the_library_refuses_them(library):
    b = kvr.Batch(i32(3), i32(2), i32(2, 8), 4, 100)
    for call in (lambda: library.cache.append(library.pool, 0, b, stream=0), lambda: library.cache.read(library.pool, 0, b, stream=0),
                 lambda: library.cache.append(library.pool, 0, b, q_out=bf(2, 2, 64), stream=0)):
        with pytest.raises(ValueError):
            call()
    assert not library.calls


def test_numbers_beyond_32_bits_are_refused_and_not_wrapped(library, monkeypatch):
    """A bound of 2^62 for "none" must not become 0, which leaves every request out."""
    b = kvr.Batch(i32(3), i32(2), i32(2, 8), 2**31 - 1, 2**31 - 1)
    assert (b.struct.max_new, b.struct.max_tokens) == (2**31 - 1, 2**31 - 1)
    for max_new, max_tokens in [(4, 1 << 62), (4, 2**32 + 100), (4, 2**31), (1 << 40, 100), (4, -2**31 - 1)]:
        with pytest.raises(ValueError):
            kvr.Batch(i32(3), i32(2), i32(2, 8), max_new, max_tokens)
    with pytest.raises(ValueError):
        kvr.rope_table(torch.zeros(10, 32, 2), first=2**32, stream=0)
    for layer in (2**32, -2**32):
        with pytest.raises(ValueError):
            library.cache.read(library.pool, layer, b, k=bf(2, 2, 64), stream=0)
        with pytest.raises(ValueError):
            library.cache.append(library.pool, layer, b, k=bf(2, 2, 64), stream=0)
        with pytest.raises(ValueError):
            library.cache.attend(library.pool, layer, b, bf(2, 4, 64), bf(2, 4, 64), i32(4), stream=0)
    assert not library.calls
    monkeypatch.undo()                                        # the library itself: a cache of 2^32 + 8 blocks is not one of 8
    for wide in (dict(num_blocks=2**32 + 8), dict(layers=2**32 + 1), dict(block_size=2**40 + 16)):
        with pytest.raises(ValueError):
            kvr.Cache(**{**dict(layers=1, kv_heads=2, head_dim=64, block_size=16, num_blocks=8), **wide})
