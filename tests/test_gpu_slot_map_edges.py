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
