"""Heads that do not fill the tiles' 64 or 128 channels, in blocks that the tile kernel loads by boxes: a box is then wider than the head, or its
second half lies partly outside, and what is outside has to read as zero."""
import numpy as np
import pytest

from test_gpu_cache import Setup, check_attend, tree

pytestmark = pytest.mark.gpu

DIMS = [(3, 5, 80, 16), (2, 4, 96, 8), (2, 8, 112, 16), (4, 4, 16, 16), (2, 8, 48, 8), (1, 8, 32, 24)]
FORMATS = [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("heads,group,dim,bs", DIMS)
@pytest.mark.parametrize("layout", [0, 1])
def test_trees(fmt, dtype, heads, group, dim, bs, layout):
    """17 to 128 rows a KV head, and more; whole tiles of context and ragged ones."""
    for new in ([20, 33, 1, 7], [64, 5, 40, 30]):
        s = Setup(fmt, heads, dim, bs, [700, 128, 0, 389], new, seed=dim + new[0], layout=layout)
        mask, seen = tree(s, np.random.default_rng(dim), empty=0.1)
        check_attend(s, heads * group, dtype, mask, seen)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("heads,group,dim,bs", DIMS)
def test_single_tokens_and_chunks(fmt, dtype, heads, group, dim, bs):
    s = Setup(fmt, heads, dim, bs, [0, 1, 300, 129, 1025], [1] * 5, seed=dim)
    check_attend(s, heads * group, dtype)
    s = Setup(fmt, heads, dim, bs, [0, 515], [300, 70], seed=dim + 1)
    check_attend(s, heads * group, dtype)
