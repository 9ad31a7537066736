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


@FMTS
@pytest.mark.parametrize("new", [[3, 0, 2], [40, 1, 30]])
@pytest.mark.parametrize("before,after", [(0, 5), (2, 0), (700, 900)])
def test_rows_of_no_request(fmt, new, before, after):
    """Before the first request's and past the last one's: zeros, as for a row
    that sees no key, and the requests' rows are what they are without them."""
    c = Case(fmt, 64, 2, 2, 16, [100, 7, 60], new=new, seed=4)
    T = before + sum(new) + after
    q = torch.full((T, 4, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    q[before:T - after] = bits_to_dev(c.qb)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    want, want_lse = c.run(decode=False)
    for with_lse in (True, False):
        out, lse = torch.full((T, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((T, 4), 7.0, device=DEV)
        ws = rfq.kv_attention_workspace(4, 64)
        rfq.rfq_kv_attention(q, c.cache, c.table, i32(c.lens), out, ws, lse=lse if with_lse else None, q_start=i32(c.start + before))
        assert rfq.rfq_workspace_status(ws) == rfq.RFQ_OK
        assert torch.equal(out[before:T - after], want)
        for rest in (slice(0, before), slice(T - after, T)):
            assert (out[rest] == 0).all()
            assert (lse[rest] == (-float("inf") if with_lse else 7.0)).all()
        if with_lse:
            assert torch.equal(lse[before:T - after], want_lse)


def test_no_request_at_all():
    c = Case(ref.FMT_MXFP4, 64, 2, 2, 16, [20], seed=5)
    q, out, lse = (torch.full(s, 7.0, dtype=d, device=DEV) for s, d in (((9, 4, 64), torch.bfloat16), ((9, 4, 64), torch.bfloat16), ((9, 4), torch.float32)))
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    for start in (0, 9):
        out.fill_(7.0)
        ws = rfq.kv_attention_workspace(4, 64)
        rfq.rfq_kv_attention(q, c.cache, none.view(0, 3), none, out, ws, lse=lse, q_start=torch.full((1,), start, dtype=torch.int32, device=DEV))
        assert rfq.rfq_workspace_status(ws) == rfq.RFQ_OK
        assert (out == 0).all() and torch.isneginf(lse).all()


@FMTS
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 4, 40])
def test_values_far_below_the_largest(fmt, D, new):
    """Values 2^24 and more below the largest of their block's dimensions may
    count as zero (HiF4 up to 32 rows: as up to 2^-21 of the largest scale);
    those of other dimensions are what they are."""
    c = Case(fmt, D, 1, 2, 16, [200], new=[new], seed=6)
    rng = np.random.default_rng(6)
    v = (rng.standard_normal((200, 1, D)) * 2.0 ** -30).astype(np.float32)
    v[7] = 0
    v[7, 0, 0] = 1000
    if D == 128:
        v[:, :, 64:] *= 2.0 ** 30
    k = torch.zeros(200, 1, D, dtype=torch.bfloat16, device=DEV)       # every key weighs the same
    slots = torch.tensor([int(c.table[0, j // 16]) * 16 + j % 16 for j in range(200)], device=DEV)
    rfq.rfq_kv_append(k, torch.from_numpy(v).to(DEV).bfloat16(), slots, c.cache)
    ko, vo = torch.empty(200, 1, D, device=DEV), torch.empty(200, 1, D, device=DEV)
    rfq.rfq_kv_read(c.cache, slots, ko, vo)
    vo = vo.double()[:, 0]
    largest = 160 if fmt == ref.FMT_HIF4 else 2.0 ** 7                 # scale of 1000: 7 x 160, 2^(9 - 2)
    block = 64 if fmt == ref.FMT_HIF4 else 32
    off = vo.abs().clone()
    off[:, block:] = 0                                                 # (blocks without a large value are exact)
    if fmt == ref.FMT_HIF4 and new * 2 <= 32:
        off[:, :block] += 2.0 ** -21 * largest
    off[7] = 0
    o, lse = c.run()
    for i in range(new):
        n = 200 - new + i + 1
        mean = vo[:n].mean(0)
        # beside it bf16's rounding and the fp32 sums; the weights are all alike, a power of two
        bound = off[:n].mean(0) + 2.0 ** -8 * mean.abs() + 2.0 ** -16 * vo[:n].abs().mean(0)
        assert ((o[i].double() - mean).abs() <= bound).all()


@FMTS
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("requests", [3, 900])
def test_a_q_start_that_descends(fmt, new, requests):
    """The requests' rows overlap, so their work is not bounded by the tokens:
    the status says so, nothing is computed, and the workspace stays usable."""
    c = Case(fmt, 64, 1, 4, 16, [600], new=[new], seed=7)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    T = 2000
    q, out = torch.zeros(T, 4, 64, dtype=torch.bfloat16, device=DEV), torch.full((T, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = rfq.kv_attention_workspace(4, 64)
    table = torch.zeros(requests, 4096, dtype=torch.int32, device=DEV)
    for start in ([T, 0] * requests, [0, T] * requests, [0] * (requests // 2) + [T] * (requests // 2) + [5] * requests):
        start = start[:requests + 1]
        rfq.rfq_kv_attention(q, c.cache, table, i32([65536] * requests), out, ws, q_start=i32(start))
        assert rfq.rfq_workspace_status(ws, clear=True) == rfq.RFQ_ERR_SHAPE
        lo, hi = start[0], start[-1]                # (what is clear of all requests may be zeros)
        assert (out[min(lo, hi):max(lo, hi)] == 7).all()
        out.fill_(7.0)
    c.check(ws=ws, decode=False)


def test_the_workspace_of_each_number_of_heads():
    """A call without heads is refused, and a short workspace still is after it."""
    c = Case(ref.FMT_MXFP4, 64, 2, 2, 16, [20], seed=8)
    q, lens = bits_to_dev(c.qb), torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    none = torch.zeros(1, 0, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_kv_attention(none, c.cache, c.table, lens, torch.empty_like(none), rfq.kv_attention_workspace(4, 64))
    assert e.value.status == rfq.RFQ_ERR_SHAPE
    with pytest.raises(ValueError):
        rfq.rfq_kv_attention(q, c.cache, c.table, lens, torch.empty_like(q), torch.zeros(64, dtype=torch.int32, device=DEV))
    for heads in (1, 4, 64):
        assert c.cache.attention_workspace_bytes(heads) == rfq.rfq_kv_attention_workspace_bytes(heads, 64) > 0
    c.check()


@FMTS
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 130, 2 ** 30, 400])
def test_windows_beyond_all_keys(fmt, window):
    """They hide nothing, also from requests with more new tokens than keys."""
    Case(fmt, 64, 2, 2, 16, [300, 5, 40], new=[10, 16, 12], seed=9).check(window=window)
    Case(fmt, 128, 1, 1, 16, [300, 5, 140], new=[450, 200, 33], seed=9).check(window=window)
    Case(fmt, 64, 1, 2, 32, [300, 140], seed=9).check(window=window)
