"""What Rope(axes=) takes for the axis of each pair: any sequence of whole numbers, by their values."""
import numpy as np
import pytest
import torch

from paper_2608_30830_b200 import kvr


@pytest.fixture
def table(monkeypatch):
    monkeypatch.setattr(kvr, "_device", lambda: (kvr._torch or kvr._use_torch()) and -1)
    return torch.zeros(10, 32, 2)


def test_sequences_of_any_kind_mean_their_numbers(table):
    want = [0] * 16 + [1] * 10 + [2] * 6
    for kind in (list, tuple, bytes, bytearray, iter, np.array, torch.tensor, lambda x: np.array(x, dtype=np.uint8), lambda x: np.array(x, dtype=np.int16), lambda x: torch.tensor(x, dtype=torch.int32)):
        rope = kvr.Rope(table, 64, axes=kind(want))
        assert rope.axes.axes == 3 and list(rope.axes.of_pair)[:32] == want and not any(list(rope.axes.of_pair)[32:])


def test_what_is_no_sequence_of_axes_is_refused(table):
    for bad in (32, np.zeros(16, dtype=np.int16), np.zeros(8, dtype=np.int32), np.zeros(4, dtype=np.int64), [0.0] * 32, [0] * 31 + [1.5], np.zeros(32), [None] * 32, "0" * 32, [0] * 31 + [256],
                [0] * 31 + [-1], [0] * 31 + [4], [0] * 33, [], np.zeros((32, 1), dtype=np.int32)):
        with pytest.raises((TypeError, ValueError)):
            kvr.Rope(table, 64, axes=bad)
