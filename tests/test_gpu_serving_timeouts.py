"""Bounded waits of the serving kernels, made to run out on purpose: a held start
keeps a kernel from issuing its first copy, so that its waits end at their limit
with nothing in flight."""
import os
import subprocess
import sys

import pytest
import torch

import serving_ref as ref
from conftest import ROOT
from gpu_util import DEV
from paper_2608_26581_gb300 import _build, rfq
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


def _in_debug_build(code):
    """Runs code against the debug build, whose kernels of few rows have a held start too."""
    code = f"import sys\nsys.path[:0] = [{ROOT!r}, {os.path.join(ROOT, 'tests')!r}]\n" + code
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=900,
                       env=dict(os.environ, RFQ_LIBRARY=_build.build(debug=True)))
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-3000:]


def few_rows():
    """Requests inside a warp's share, over many warps and CTAs, and without
    keys.  The parts of those that are shared are joined all the same, so the
    workspace serves the next call."""
    lens = [3000, 100, 0, 20000, 17]
    for fmt in (ref.FMT_MXFP4, ref.FMT_HIF4):
        for D in (64, 128):
            for new in (1, 4):
                c = Case(fmt, D, 2, 4, 16, lens, new=[new] * len(lens), seed=14)
                ws = rfq.kv_attention_workspace(8, D)
                for _ in range(2):
                    out, lse, status = _held(c, ws)
                    assert status == rfq.RFQ_ERR_TIMEOUT
                    assert torch.isnan(out.float()).all() and torch.isnan(lse).all()
                    c.check(ws=ws, decode=False)
                ws[2] = 1                 # an open gate
                ws[3] = 1
                c.check(ws=ws, decode=False)


def test_attention_of_few_rows():
    _in_debug_build("import test_gpu_serving_timeouts as t\nt.few_rows()\n")


def matvec():
    """Of every number of rows, with K in one share, over a cluster, and in
    phases of what of x fits; the next call is right."""
    rng = torch.Generator(device=DEV)
    rng.manual_seed(0)
    for fmt in (rfq.RFQ_FMT_MXFP4, rfq.RFQ_FMT_HIF4):
        for M, K, N in ((1, 512, 40), (2, 4096, 5000), (4, 12288, 300), (8, 2048, 700), (13, 12288, 300), (32, 12288, 130)):
            w = rfq.empty_qtensor(fmt, rfq.RFQ_SCALE_MMA, N, K)
            rfq.rfq_quantize_weight(torch.randn(K, N, generator=rng, device=DEV).bfloat16(), w)
            x = torch.randn(M, K, generator=rng, device=DEV).bfloat16()
            want, y = torch.empty(M, N, device=DEV), torch.zeros(M, N, device=DEV)
            rfq.rfq_matvec(x, w, want)
            os.environ["RFQ_DEBUG_HOLD_US"] = "2000"
            rfq.rfq_matvec(x, w, y)
            torch.cuda.synchronize()
            del os.environ["RFQ_DEBUG_HOLD_US"]
            assert torch.isnan(y).all()
            rfq.rfq_matvec(x, w, y)
            assert torch.isfinite(want).all() and torch.equal(y, want)


def test_matvec():
    _in_debug_build("import test_gpu_serving_timeouts as t\nt.matvec()\n")
