"""Pairs sorted by expert, rows brought to their groups and back, quantized on
the way, and the gradients: places and copies exactly, sums within bounds
counted from fp32's roundings (tests/moe_ref.py)."""
import numpy as np
import pytest
import torch

import moe_ref
from gpu_util import DEV, guarded_empty, guarded_full, qtensor_host
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
U = moe_ref.U


def _ids(seed, T, k, E, kind="spread"):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":                                  # every pair of one expert
        return torch.full((T, k), E - 1, dtype=I32)
    if kind == "none":
        return torch.full((T, k), -1, dtype=I32)
    like = torch.randn(T, E, generator=g) + torch.randn(E, generator=g)
    ids = like.topk(k, -1).indices.int()
    if kind == "holes":
        ids[torch.rand(T, k, generator=g) < 0.2] = -1
        ids[torch.rand(T, k, generator=g) < 0.05] = E  # foreign ids
        ids[T - T // 4:] = -1
    return ids


def _sort(ids, E, align, rows):
    T, k = ids.shape
    off, row_of, pair_of = (guarded_full(s, 99, I32) for s in ((E + 1,), (T, k), (rows,)))
    ws = torch.zeros(64, dtype=I32, device=DEV)
    rfq.rfq_moe_sort(ids.to(DEV), off, row_of, pair_of, ws, align=align)
    return off, row_of, pair_of, rfq.rfq_workspace_status(ws)


@pytest.mark.parametrize("align", [1, 7, 128])
@pytest.mark.parametrize("kind", ["spread", "holes", "one", "none"])
@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 128), (5, 3, 4), (61, 8, 128), (512, 8, 64), (700, 6, 60), (1025, 4, 256), (4100, 8, 128),
                                   (600, 32, 33)])
def test_sort(T, k, E, kind, align):
    ids = _ids(T, T, k, E, kind)
    rows = rfq.rfq_moe_rows(T, k, E, align) + 5
    off, row_of, pair_of, status = _sort(ids, E, align, rows)
    want = moe_ref.sort(ids, E, align, rows)
    assert status == rfq.RFQ_OK and want[3]
    for a, b in zip((off, row_of, pair_of), want):
        assert torch.equal(a.cpu(), b)


def test_sort_up_to_31_bits():
    """As many pairs as are taken: the rows behind the last group start just below 2^31."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T = 2 ** 31 - 2
    # (one array, pair_of last: 2^31 elements before a row of pair_of lies row_of)
    words = torch.zeros(3 * (2 ** 31 + 64), dtype=I32, device=DEV)
    ids, row_of, pair_of = (w[:n] for w, n in zip(words.view(3, -1), (T, T, T + 1)))
    off, ws = torch.zeros(2, dtype=I32, device=DEV), torch.zeros(64, dtype=I32, device=DEV)
    rfq.rfq_moe_sort(ids.view(T, 1), off, row_of.view(T, 1), pair_of, ws, align=1)
    assert rfq.rfq_workspace_status(ws) == rfq.RFQ_OK and off.tolist() == [0, T] and pair_of[T].item() == -1
    for a in range(0, T, 2 ** 28):
        want = torch.arange(a, min(T, a + 2 ** 28), dtype=I32, device=DEV)
        assert torch.equal(row_of[a:a + 2 ** 28], want) and torch.equal(pair_of[a:min(T, a + 2 ** 28)], want)
    assert (words.view(3, -1)[1, T:] == 0).all() and (words.view(3, -1)[2, T + 1:] == 0).all()


def test_sort_of_many_pairs():
    """262144 pairs over one cluster, against a stable sort."""
    T, k, E = 32768, 8, 128
    ids = _ids(9, T, k, E, "holes")
    rows = rfq.rfq_moe_rows(T, k, E, 128)
    off, row_of, pair_of, status = _sort(ids, E, 128, rows)
    flat = ids.flatten().numpy()
    ok = (flat >= 0) & (flat < E)
    order = np.argsort(np.where(ok, flat, E), kind="stable")[:ok.sum()]
    size = np.bincount(flat[ok], minlength=E)
    start = np.concatenate([[0], np.cumsum(-(-size // 128) * 128)])
    place = start[flat[order]] + np.arange(len(order)) - (np.cumsum(size) - size)[flat[order]]
    want_row, want_pair = np.full(T * k, -1), np.full(rows, -1)
    want_row[order], want_pair[place] = place, order
    assert status == rfq.RFQ_OK and np.array_equal(off.cpu().numpy(), start)
    assert np.array_equal(row_of.cpu().numpy().ravel(), want_row) and np.array_equal(pair_of.cpu().numpy(), want_pair)


@pytest.mark.parametrize("rows", [0, 1, 100, 128, 300, 511, 640])
@pytest.mark.parametrize("align", [1, 128])
def test_sort_without_room(rows, align):
    """Too few rows: the pairs that fit are served, the status says so."""
    ids = _ids(2, 100, 4, 9)
    off, row_of, pair_of, status = _sort(ids, 9, align, rows)
    want = moe_ref.sort(ids, 9, align, rows)
    assert (status == rfq.RFQ_OK) == want[3]
    assert status in (rfq.RFQ_OK, rfq.RFQ_ERR_SHAPE)
    for a, b in zip((off, row_of, pair_of), want):
        assert torch.equal(a.cpu(), b)


def _maps(seed, T, k, E, align, kind, extra=0):
    ids = _ids(seed, T, k, E, kind)
    rows = rfq.rfq_moe_rows(T, k, E, align) + extra
    _, row_of, pair_of, _ = moe_ref.sort(ids, E, align, rows)
    return rows, row_of, pair_of


CASES = [(1, 1, 1, 1, "spread"), (1, 8, 16, 128, "spread"), (5, 3, 4, 1, "holes"), (61, 8, 128, 16, "holes"), (130, 6, 60, 1, "spread"),
         (40, 32, 64, 7, "spread"), (33, 2, 5, 128, "one"), (9, 4, 8, 16, "none")]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [1, 2, 6, 8, 12, 33, 100, 128, 130, 1000, 1030, 2048, 4104])
@pytest.mark.parametrize("T,k,E,align,kind", CASES)
def test_rows_there_and_back(T, k, E, align, kind, dim, dtype):
    rows, row_of, pair_of = _maps(T + dim, T, k, E, align, kind, extra=3)
    g = torch.Generator().manual_seed(dim)
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    R, P = row_of.to(DEV), pair_of.to(DEV)
    pair = pair_of.long()
    there = pair >= 0
    # there
    x = rnd(T, dim)
    out = guarded_full((rows, dim), float("nan"), dtype)
    rfq.rfq_moe_gather(x.to(DEV), R, out, pair_of=P)
    want = torch.where(there[:, None], x[pair.clamp_min(0) // k], 0)
    assert torch.equal(out.cpu(), want)
    some = guarded_full((rows, dim), 7.0, dtype)
    rfq.rfq_moe_gather(x.to(DEV), R, some)
    assert torch.equal(some.cpu(), torch.where(there[:, None], want, torch.full_like(want, 7.0)))
    # back
    y, w = rnd(rows, dim), torch.randn(T, k, generator=g)
    terms = torch.where((row_of >= 0)[..., None], y.double()[row_of.long().clamp_min(0)], 0.0)
    for weights in (w, None):
        back = guarded_full((T, dim), float("nan"), dtype)
        rfq.rfq_moe_combine(y.to(DEV), R, back, weights=None if weights is None else weights.to(DEV))
        each = terms if weights is None else terms * weights.double()[..., None]
        total = each.sum(1)
        e = (k + 1) * U * each.abs().sum(1)            # a product and k additions at most
        assert ((back.double().cpu() - total).abs() <= e + moe_ref.half_step(dtype) * (total.abs() + e)).all()
    # gradients
    dout = rnd(T, dim)
    dy, dw = guarded_full((rows, dim), float("nan"), dtype), guarded_full((T, k), float("nan"), F32)
    rfq.rfq_moe_combine_grad(dout.to(DEV), y.to(DEV), R, w.to(DEV), dy, dw, pair_of=P)
    want = torch.where(there[:, None], dout.double()[pair.clamp_min(0) // k] * w.double().flatten()[pair.clamp_min(0)][:, None], 0.0)
    # (a product of fp32, then the type's rounding)
    assert ((dy.double().cpu() - want).abs() <= (moe_ref.half_step(dtype) + 2 * U) * want.abs() + 2.0 ** -140).all()
    dots = terms * dout.double()[:, None]
    # a lane's own products and additions, then five over lanes
    e = (2 * -(-dim // 32) + 8) * U * dots.abs().sum(-1)
    assert ((dw.double().cpu() - dots.sum(-1)).abs() <= e).all()
    # dy in the place of y, without clearing: the same values at the rows of pairs
    same, dw2 = y.to(DEV), torch.empty_like(dw)
    rfq.rfq_moe_combine_grad(dout.to(DEV), same, R, w.to(DEV), same, dw2)
    assert torch.equal(dw2, dw) and torch.equal(same.cpu()[there], dy.cpu()[there]) and torch.equal(same.cpu()[~there], y[~there])


def test_rows_that_lie_apart():
    """Token rows with strides, also such as no 16-byte access fits."""
    rows, row_of, pair_of = _maps(1, 21, 4, 8, 16, "holes")
    R, P = row_of.to(DEV), pair_of.to(DEV)
    w = torch.rand(21, 4, device=DEV)
    for dtype in (BF16, F32):
        for stride in (96, 97):
            base = torch.randn(21, stride, device=DEV).to(dtype)
            x = base[:, :64]
            a, b = torch.empty(rows, 64, dtype=dtype, device=DEV), torch.empty(rows, 64, dtype=dtype, device=DEV)
            rfq.rfq_moe_gather(x, R, a, pair_of=P)
            rfq.rfq_moe_gather(x.contiguous(), R, b, pair_of=P)
            assert torch.equal(a, b)
            out = torch.zeros(21, stride, dtype=dtype, device=DEV)
            want = torch.empty(21, 64, dtype=dtype, device=DEV)
            rfq.rfq_moe_combine(a, R, out[:, :64], weights=w)
            rfq.rfq_moe_combine(a, R, want, weights=w)
            assert torch.equal(out[:, :64], want) and (out[:, 64:] == 0).all()
            d1, d2 = torch.empty_like(a), torch.empty_like(a)
            w1, w2 = torch.empty_like(w), torch.empty_like(w)
            rfq.rfq_moe_combine_grad(x, a, R, w, d1, w1, pair_of=P)
            rfq.rfq_moe_combine_grad(x.contiguous(), a, R, w, d2, w2, pair_of=P)
            assert torch.equal(d1, d2) and torch.allclose(w1, w2, rtol=1e-5, atol=1e-5)


def test_foreign_rows_are_skipped():
    """Rows outside the stacked matrix are neither written nor read."""
    T, k, rows, dim = 6, 3, 10, 72
    row_of = torch.tensor([[0, -1, 10], [2 ** 31 - 1, 3, -2 ** 31], [9, 4, 5], [11, 12, 13], [-7, 1, 2], [6, 7, 8]], dtype=I32)
    x = torch.randn(T, dim)
    out = guarded_full((rows, dim), 5.0, F32)
    rfq.rfq_moe_gather(x.to(DEV), row_of.to(DEV), out)
    want = torch.full((rows, dim), 5.0)
    for t in range(T):
        for r in row_of[t].tolist():
            if 0 <= r < rows:
                want[r] = x[t]
    assert torch.equal(out.cpu(), want)
    back = torch.empty(T, dim, device=DEV)
    rfq.rfq_moe_combine(out, row_of.to(DEV), back)
    assert (back[3] == 0).all() and torch.equal(back[1].cpu(), x[1])
    dy, dw = guarded_full((rows, dim), 5.0, F32), torch.empty(T, k, device=DEV)
    rfq.rfq_moe_combine_grad(x.to(DEV), out, row_of.to(DEV), torch.ones(T, k, device=DEV), dy, dw)
    assert torch.equal(dy.cpu(), want) and (dw.cpu()[(row_of < 0) | (row_of >= rows)] == 0).all()
    xb = torch.randn(T, 128, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    q = rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, rows, 128)
    q.codes.fill_(0x33)
    rfq.rfq_moe_quantize(xb, row_of.to(DEV), q)
    ref = rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, T, 128)
    rfq.rfq_quantize_act(xb, ref, None, mode=rfq.RFQ_FALLBACK_NONE)
    codes, want = qtensor_host(q)[0], qtensor_host(ref)[0]
    for t in range(T):
        for r in row_of[t].tolist():
            if 0 <= r < rows:
                assert np.array_equal(codes[r], want[t])


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("clear", [False, True])
@pytest.mark.parametrize("T,k,E,align,kind", CASES)
@pytest.mark.parametrize("dim", [128, 640, 2048, 1152])
def test_quantize(orc, T, k, E, align, kind, dim, clear, residual):
    """Bytes of the oracle's encoder at the rows of pairs, zeros (or what was
    there) at the others, zero scales in the layout's padding."""
    rows, row_of, pair_of = _maps(T + dim, T, k, E, align, kind, extra=3)
    g = torch.Generator().manual_seed(dim + T)
    x = (torch.randn(T, dim + 8, generator=g) * (1 + 50 * (torch.rand(dim + 8, generator=g) < 0.02).float())).bfloat16()
    x[:, 3] *= 1e-30
    x[T // 2, :64] = 0
    make = lambda: rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, rows, dim)  # noqa: E731
    xq, xr = make(), make() if residual else None
    for q in (xq, xr):
        if q is not None:
            q.codes.fill_(0x5A)
            q.scales.fill_(0x5A)
    rfq.rfq_moe_quantize(x.to(DEV)[:, :dim], row_of.to(DEV), xq, xr, pair_of=pair_of.to(DEV) if clear else None)
    o = orc.quantize_act(x[:, :dim].contiguous().view(torch.int16).numpy().view(np.uint16))
    there = pair_of.numpy() >= 0
    token = pair_of.numpy()[there] // k
    for q, name in ((xq, "main"), (xr, "res")):
        if q is None:
            continue
        codes, scales = qtensor_host(q)
        assert np.array_equal(codes[there], o[name + "_codes"][token]) and np.array_equal(scales[there], o[name + "_scales"][token])
        left = 0 if clear else 0x5A
        assert (codes[~there] == left).all() and (scales[~there] == left).all()
        # the layout's rows behind the last
        from gpu_util import mma_scale_to_rowmajor
        padded = -(-rows // 128) * 128
        assert (mma_scale_to_rowmajor(q.scales.cpu().numpy(), padded, dim)[rows:] == 0).all()


def test_nothing_to_do():
    e = lambda *s, t=F32: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
    off, ws = torch.full((5,), 9, dtype=I32, device=DEV), torch.zeros(64, dtype=I32, device=DEV)
    pair = torch.full((16,), 9, dtype=I32, device=DEV)
    rfq.rfq_moe_sort(e(0, 2, t=I32), off, e(0, 2, t=I32), pair, ws, align=8)
    assert (off == 0).all() and (pair == -1).all()
    out = torch.full((16, 40), 3.0, device=DEV)
    rfq.rfq_moe_gather(e(0, 40), e(0, 2, t=I32), out, pair_of=pair)
    assert (out == 0).all()
    rfq.rfq_moe_gather(e(0, 40), e(0, 2, t=I32), e(0, 40), pair_of=e(0, t=I32))
    rfq.rfq_moe_combine(out, e(0, 2, t=I32), e(0, 40))
    none = torch.full((3, 2), -1, dtype=I32, device=DEV)
    back = torch.full((3, 40), 3.0, device=DEV)
    rfq.rfq_moe_combine(e(0, 40), none, back)
    assert (back == 0).all()
    dw = torch.full((3, 2), 3.0, device=DEV)
    rfq.rfq_moe_combine_grad(back, e(0, 40), none, e(3, 2), e(0, 40), dw)
    assert (dw == 0).all()
