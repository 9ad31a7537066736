"""rfq_slot_map at the ends of its ranges: drops of any size, lengths past 32
bits, and every number of requests from a fresh process."""
import os
import subprocess
import sys

import numpy as np
import pytest

from conftest import ROOT
from test_gpu_slot_map import _check, _run

pytestmark = pytest.mark.gpu
LEAST = -2 ** 31


@pytest.mark.parametrize("drop", [LEAST, LEAST + 1, -41, -40])
@pytest.mark.parametrize("alias", [False, True])
def test_a_request_that_drops_all(drop, alias):
    """Its pages go back, its length is 0, and another request takes the pages
    in the same step."""
    _check([40, 5, 16, 0], [drop, 60, drop, drop], 16, 8, [50, 51, 0, 0, 0, 0], 1, 60, alias=alias)


@pytest.mark.parametrize("R", [2004, 2005, 2025, 2026, 2047, 2048])
def test_requests_of_a_first_call(R):
    """Every number of requests works in a process that has made no larger call."""
    code = f"""
import sys
sys.path[:0] = [{ROOT!r}, {os.path.join(ROOT, "tests")!r}]
from test_gpu_slot_map import _check
_check([3, 20] * {R // 2} + [3] * {R % 2}, [1] * {R}, 16, 4, list(range({R})), {R}, {R})
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("added", [4, 5, 2 ** 31 - 1])
def test_a_length_past_32_bits(added):
    """It does not fit, however wide the table: nothing taken, the length kept."""
    page, cached = 2 ** 30, 2 ** 31 - 4
    table = np.array([[3, 4, -1, -1], [5, -1, -1, -1]], np.int32)
    t, free, count, lengths, start, slots, pos, bad = _run([cached, 7], [added, 1], page, table, [8, 9], 2, 6)
    np.testing.assert_array_equal(t, table)
    assert free.tolist() == [8, 9] and count.tolist() == [2] and lengths.tolist() == [cached, 8] and bad
    assert start.tolist() == [0, added, min(added + 1, 2 ** 31 - 1)]
    assert slots[:min(added, 6)].tolist() == [-1] * min(added, 6)
    if added < 6:
        assert slots[added] == 5 * page + 7 and pos[added] == 7


def test_the_longest_request():
    page, cached = 2 ** 30, 2 ** 31 - 4
    table = np.array([[3, 4]], np.int32)
    t, free, count, lengths, start, slots, pos, bad = _run([cached], [3], page, table, [8], 1, 3)
    assert count.tolist() == [1] and lengths.tolist() == [2 ** 31 - 1] and not bad
    assert pos.tolist() == [cached, cached + 1, cached + 2] and slots.tolist() == [4 * page + p - page for p in pos.tolist()]
