"""rfq_slot_map at the ends of its ranges: drops of any size, lengths past 32
bits, and every number of requests from a fresh process."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT
from test_gpu_slot_map import _check

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
