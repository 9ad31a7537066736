"""rfq_kv_attention at the ends of what its arguments may be."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import DEV
from paper_2608_26581_gb300 import rfq
from test_gpu_kv_attention import FMTS, Case, bits_to_dev

pytestmark = pytest.mark.gpu


@FMTS
@pytest.mark.parametrize("new", [[300], [300, 1, 7]])
def test_a_table_for_many_keys(fmt, new):
    """A prompt in tiles of 128 rows, with room for 2^26 keys a request."""
    c = Case(fmt, 64, 8, 8, 64, [400] * len(new), new=new, seed=3)
    wide = torch.full((len(new), 2 ** 20), -1, dtype=torch.int32, device=DEV)
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide
    c.check()
