"""Attention raises its kernels' limit of shared memory once on every device that is current in a call, not once a process."""
from paper_2608_30830_b200 import kvr


def test_every_device_gets_its_own():
    assert kvr.test_once([0, 0, 1, 0, 1, 63, 63, 7], [0] * 8) == ([0] * 8, 4)


def test_a_failure_is_returned_and_tried_again():
    # device 0 fails twice, then is done; device 1 is not touched by that
    assert kvr.test_once([0, 1, 0, 0, 0, 1], [2, 0, 3, 0, 9, 9]) == ([2, 0, 3, 0, 0, 0], 4)


def test_devices_that_no_bit_stands_for():
    assert kvr.test_once([64, 64, -1, 64, 0, 0], [0, 5, 0, 0, 0, 0]) == ([0, 5, 0, 0, 0, 0], 5)
