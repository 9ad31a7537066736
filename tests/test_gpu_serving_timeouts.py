"""Bounded waits of the serving kernels, made to run out on purpose: a held start
keeps a kernel from issuing its first copy, so that its waits end at their limit
with nothing in flight."""
import pytest
import torch

from gpu_util import DEV
from paper_2608_26581_gb300 import rfq
from test_gpu_kv_attention import FMTS, Case, bits_to_dev

pytestmark = pytest.mark.gpu


def _held(c, ws):
    """The outputs of a call whose start stays held for 20 ms."""
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    words = ws[:4]
    words[1] = 20000
    words[2] = 1
    q, out = bits_to_dev(c.qb), torch.zeros(c.qb.shape, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros(c.qb.shape[:2], device=DEV)
    rfq.rfq_kv_attention(q, c.cache, c.table, i32(c.lens), out, ws, lse=lse, q_start=i32(c.start))
    status = rfq.rfq_workspace_status(ws)
    words.zero_()
    return out, lse, status


@FMTS
def test_attention_tiles_leave_nan_in_both_outputs(fmt):
    c = Case(fmt, 128, 2, 4, 16, [3000, 100], new=[100, 30], seed=13)
    ws = rfq.kv_attention_workspace(8, 128)
    out, lse, status = _held(c, ws)
    assert status == rfq.RFQ_ERR_TIMEOUT
    assert torch.isnan(out.float()).all() and torch.isnan(lse).all()
    c.check(ws=ws)
