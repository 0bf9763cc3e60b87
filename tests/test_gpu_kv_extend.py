"""A step whose returned pages would not fit the ring beside those it holds."""

import pytest

from tests.test_gpu_kv import run_extend

pytestmark = pytest.mark.gpu


def test_pages_that_would_come_back_over_those_taken_are_refused():
    """Two pages are held and three more are said to be free, of four: returning both would
    write where the step takes its pages from."""
    page, table, ring = 16, [[0, 1, -5], [-5, -5, -5]], [2, 3, 1, -1]
    got = run_extend([20, 0], [0, 40], 0, 3, table, ring, page, 40)
    assert got["result"] == [-1, 0, 0, 0] and got["lengths"] == [20, 0] and got["pos"] == [0, 3]
    assert got["table"] == table and got["ring"] == ring and got["slots"] == [-1] * 40
    # the same step of a ring that tells the truth
    got = run_extend([20, 0], [0, 30], 0, 2, table, ring, page, 40)
    assert got["result"] == [0, 30, 2, 2] and got["pos"] == [2, 2]
    assert got["table"][1][:2] == [2, 3] and got["ring"] == [2, 3, 0, 1]
