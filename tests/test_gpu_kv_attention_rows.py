"""rfq_kv_attention with many rows a request (new tokens times query heads of a
key head): the tiles of 128 rows by 128 keys, and batches that mix both."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import DEV
from paper_2608_26581_gb300 import rfq
from paper_2608_26581_gb300.synth import bf16_bits_to_f32, f32_to_bf16_bits
from test_gpu_kv_attention import FMTS, Case, bits_to_dev

pytestmark = pytest.mark.gpu


@FMTS
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,new", [(1, [65, 127, 128, 129, 300]), (3, [22, 43, 100, 171, 1]), (8, [9, 16, 17, 0, 40])])
def test_rows_around_a_tile(fmt, D, G, new):
    """65 to 513 rows: tiles that end inside a token; keys that end inside a
    chunk; a request of one token or none beside them."""
    Case(fmt, D, 2, G, 16, [65, 255, 256, 300, 513], new=new, seed=G).check()


@FMTS
@pytest.mark.parametrize("page", [16, 48, 64, 128, 384])
def test_pages(fmt, page):
    Case(fmt, 128, 2, 4, page, [127, 128, 129, 700], new=[20, 33, 64, 50], seed=page).check()


@FMTS
@pytest.mark.parametrize("window", [1, 16, 100, 129, 1000])
@pytest.mark.parametrize("page", [16, 128])
def test_windows(fmt, window, page):
    Case(fmt, 64, 2, 2, page, [200, 517, 90], new=[150, 80, 70], seed=window).check(window=window)
    Case(fmt, 128, 1, 4, page, [900], new=[300], seed=window).check(window=window)


@FMTS
def test_rows_before_the_first_key(fmt):
    """More new tokens than keys: whole tiles that see nothing."""
    Case(fmt, 128, 2, 1, 16, [3, 0, 130], new=[300, 70, 200], seed=1).check()


@FMTS
def test_one_token_of_many_heads(fmt):
    """Single tokens reach a tile's rows through their heads alone."""
    Case(fmt, 64, 2, 80, 16, [1, 0, 129, 400], seed=2).check()
    Case(fmt, 128, 1, 130, 32, [257, 5], seed=3).check(decode=False)


@FMTS
def test_split_over_ctas(fmt):
    Case(fmt, 128, 1, 2, 64, [20000, 40], new=[50, 33], seed=4).check()
    Case(fmt, 64, 2, 1, 16, [9001], new=[140], seed=5).check()


def test_many_requests():
    rng = np.random.default_rng(0)
    new = rng.choice([0, 1, 2, 70, 130], 60).tolist()
    Case(ref.FMT_MXFP4, 64, 1, 1, 16, rng.integers(0, 300, 60).tolist(), new=new, seed=6).check()


def test_many_requests_some_of_many_tiles():
    """More requests than a CTA's warps take one by one, among them some with
    more tiles than one lane counts."""
    new = [1, 0, 300, 2, 9] * 10
    Case(ref.FMT_HIF4, 64, 2, 4, 32, [(17 * i) % 420 for i in range(50)], new=new, seed=14).check()


@FMTS
def test_scales_span_many_octaves(fmt):
    """Values, and with them the running powers of two, grow and fall by 2^20
    between tokens; so do the scores, through the queries."""
    c = Case(fmt, 128, 2, 4, 16, [600, 300], new=[40, 20], seed=7, vspread=10)
    c.check()
    q = bf16_bits_to_f32(c.qb) * (2.0 ** np.linspace(-100, 3, c.qb.shape[1]))[None, :, None]
    q[1, 3] = 0
    c.check(qbits=f32_to_bf16_bits(q.astype(np.float32)))


@FMTS
def test_keys_span_many_octaves(fmt):
    """Keys 2^12 apart in one tile and between tiles, which f16 holds exactly
    beside the largest scale."""
    rng = np.random.default_rng(8)
    c = Case(fmt, 64, 1, 2, 16, [500], new=[60], seed=8)
    k = rng.standard_normal((500, 1, 64)) * 2.0 ** rng.integers(-12, 1, (500, 1, 1))
    v = rng.standard_normal((500, 1, 64))
    slots = torch.tensor([int(c.table[0, j // 16]) * 16 + j % 16 for j in range(500)], device=DEV)
    rfq.rfq_kv_append(bits_to_dev(f32_to_bf16_bits(k.astype(np.float32))), bits_to_dev(f32_to_bf16_bits(v.astype(np.float32))),
                      slots, c.cache)
    ko, vo = torch.empty(500, 1, 64, device=DEV), torch.empty(500, 1, 64, device=DEV)
    rfq.rfq_kv_read(c.cache, slots, ko, vo)
    c.keys, c.values = [ko.double().cpu().numpy()], [vo.double().cpu().numpy()]
    c.vmax = np.abs(c.values[0]).max()
    c.check()


def test_scale_zero_and_negative():
    c = Case(ref.FMT_HIF4, 64, 1, 4, 16, [177], new=[40], seed=9)
    c.check(scale=0.0)
    c.check(scale=-0.3)


def test_same_bits_twice_and_workspace_reuse():
    c = Case(ref.FMT_MXFP4, 128, 2, 4, 16, [3000, 100, 900], new=[100, 1, 30], seed=10)
    d = Case(ref.FMT_HIF4, 128, 2, 4, 16, [3000], new=[20], seed=11)
    ws = rfq.kv_attention_workspace(8, 128)
    a = c.run(ws=ws)
    d.check(ws=ws)
    for _ in range(3):
        b = c.run(ws=ws)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@FMTS
def test_a_wait_that_runs_out(fmt):
    """The held start (word 2 set, word 3 zero) keeps the copies from starting:
    every wait of the kernel ends at its limit, none of its copies or MMAs in
    flight.  The status tells, the rows are NaN, and once the words are cleared
    the workspace serves the next call."""
    c = Case(fmt, 128, 2, 4, 16, [3000, 100], new=[100, 30], seed=13)
    ws = rfq.kv_attention_workspace(8, 128)
    words = ws[:4]
    words[1] = 20000
    words[2] = 1
    q, out = bits_to_dev(c.qb), torch.zeros(c.qb.shape, dtype=torch.bfloat16, device=DEV)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    rfq.rfq_kv_attention(q, c.cache, c.table, i32(c.lens), out, ws, q_start=i32(c.start))
    assert rfq.rfq_workspace_status(ws) == rfq.RFQ_ERR_TIMEOUT
    assert torch.isnan(out.float()).all()
    words.zero_()
    c.check(ws=ws)
    words[2] = 1                      # an open gate
    words[3] = 1
    c.check(ws=ws)


def test_bad_device_sizes_set_the_status():
    c = Case(ref.FMT_MXFP4, 64, 1, 2, 16, [150, 30], new=[60, 40], seed=12, poison=False)
    q = bits_to_dev(c.qb)

    def status(table, lens, start):
        ws, out = rfq.kv_attention_workspace(2, 64), torch.zeros_like(q)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        rfq.rfq_kv_attention(q, c.cache, table, i32(lens), out, ws, q_start=i32(start))
        return rfq.rfq_workspace_status(ws)
    assert status(c.table, [150, 30], [0, 60, 100]) == rfq.RFQ_OK
    assert status(c.table, [161, 30], [0, 60, 100]) == rfq.RFQ_ERR_SHAPE
    assert status(torch.full_like(c.table, 2 ** 30), [150, 30], [0, 60, 100]) == rfq.RFQ_ERR_SHAPE
    assert status(torch.full_like(c.table, -1), [150, 30], [0, 60, 100]) == rfq.RFQ_ERR_SHAPE
    assert status(c.table, [150, 30], [0, 60, 200]) == rfq.RFQ_ERR_SHAPE
