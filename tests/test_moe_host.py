"""Host-side checks of the entry points around a mixture-of-experts block:
every refusal comes before any device work (the pointers below are not device
memory), and the references agree with derivatives taken by autograd."""
import ctypes

import pytest
import torch

import moe_ref
from fake_cuda import FakeCuda
from paper_2608_26581_gb300 import rfq

E_ARG, E_SHAPE, E_ALIGN, E_UNSUPPORTED = rfq.RFQ_ERR_INVALID_ARG, rfq.RFQ_ERR_SHAPE, rfq.RFQ_ERR_ALIGNMENT, rfq.RFQ_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    from paper_2608_26581_gb300 import _build
    _build.build()
    return rfq.load_library()


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeCuda(tmp_path_factory.mktemp("fake"))


def _checks(f, good, wrong):
    """Every (argument, value): the status that the call gives with it."""
    for status, cases in wrong.items():
        for i, v in cases:
            a = list(good)
            a[i] = v
            assert f(*a) == status, (i, v)


def test_norm_checks(lib):
    good = [16, 256, 64, 16, 256, 64, 1, 3, 4, 64, 0, 1e-6, 16, 16, 1, 16, 16, None]
    _checks(lib.rfq_norm, good, {
        E_ARG: [(0, None), (3, None), (6, 2), (10, 2), (11, float("nan")), (11, -1.0), (14, 2)],
        E_SHAPE: [(1, -1), (2, -1), (4, -1), (5, -1), (7, -1), (7, 2 ** 31), (8, 0), (9, 0), (9, 16385)],
        E_ALIGN: [(0, 24), (3, 8), (12, 8), (13, 4), (15, 2), (16, 6)]})


def test_norm_grad_checks(lib):
    good = [16, 256, 64, 16, 256, 64, 16, 256, 64, 1, 3, 4, 64, 0, 16, 16, 16, 1, 16, 16, 16, None]
    _checks(lib.rfq_norm_grad, good, {
        E_ARG: [(0, None), (3, None), (6, None), (14, None), (15, None), (20, None), (9, 2), (13, 2), (17, -1)],
        E_SHAPE: [(1, -1), (5, -1), (8, -1), (10, -1), (10, 2 ** 30), (11, 0), (12, 0), (12, 16385)],
        E_ALIGN: [(0, 24), (3, 8), (6, 8), (14, 2), (15, 2), (16, 8), (18, 2), (19, 2), (20, 8)]})
    assert lib.rfq_norm_grad_workspace_bytes(0) == 0 and lib.rfq_norm_grad_workspace_bytes(16385) == 0


def test_route_checks(lib):
    good = [16, 128, 0, 3, 128, 8, 1, 16, 16, None]
    _checks(lib.rfq_route, good, {
        E_ARG: [(0, None), (7, None), (8, None), (2, 2)],
        E_SHAPE: [(1, -1), (3, -1), (3, 2 ** 30), (4, 0), (4, 257), (4, 7), (5, 0), (5, 33)],
        E_ALIGN: [(0, 8), (7, 2), (8, 6)]})
    good = [16, 128, 0, 3, 128, 8, 1, 16, 16, 16, 128, None]
    _checks(lib.rfq_route_grad, good, {
        E_ARG: [(0, None), (7, None), (8, None), (9, None), (2, 2)],
        E_SHAPE: [(1, -1), (3, -1), (4, 257), (4, 7), (5, 0), (10, -1)],
        E_ALIGN: [(0, 8), (7, 2), (8, 6), (9, 8)]})


def test_sort_checks(lib):
    good = [16, 3, 8, 128, 128, 16, 16, 16, 4096, 16, None]
    _checks(lib.rfq_moe_sort, good, {
        E_ARG: [(0, None), (5, None), (6, None), (7, None), (9, None)],
        E_SHAPE: [(1, -1), (1, 2 ** 28), (2, 0), (2, 33), (3, 0), (3, 257), (4, 0), (4, 4097), (8, -1), (8, 2 ** 31)],
        E_ALIGN: [(0, 2), (5, 6), (6, 2), (7, 2), (9, 8)]})
    assert lib.rfq_moe_rows(0, 8, 128, 128) == 0 and lib.rfq_moe_rows(1, 8, 128, 128) == 8 * 128
    assert lib.rfq_moe_rows(4096, 8, 128, 128) == 32768 + 127 * 128 and lib.rfq_moe_rows(5, 3, 4, 1) == 15
    for bad in ((-1, 8, 128, 128), (1, 0, 128, 128), (1, 8, 257, 128), (1, 8, 128, 0)):
        assert lib.rfq_moe_rows(*bad) == -1


def test_rows_checks(lib):
    good = [16, 64, 1, 3, 64, 16, 8, 16, 16, 24, None]
    _checks(lib.rfq_moe_gather, good, {
        E_ARG: [(0, None), (5, None), (8, None), (2, 2)],
        E_SHAPE: [(1, -1), (3, -1), (4, 0), (4, 65537), (6, 0), (6, 33), (9, -1), (9, 2 ** 31)],
        E_ALIGN: [(0, 8), (5, 2), (7, 2), (8, 8)]})
    good = [16, 1, 24, 64, 16, 16, 3, 8, 16, 64, None]
    _checks(lib.rfq_moe_combine, good, {
        E_ARG: [(0, None), (4, None), (8, None), (1, 2)],
        E_SHAPE: [(2, -1), (3, 0), (6, -1), (7, 0), (7, 33), (9, -1)],
        E_ALIGN: [(0, 8), (4, 2), (5, 2), (8, 8)]})
    good = [16, 64, 16, 1, 24, 64, 16, 16, 16, 3, 8, 16, 16, None]
    _checks(lib.rfq_moe_combine_grad, good, {
        E_ARG: [(0, None), (2, None), (6, None), (8, None), (11, None), (12, None), (3, 2)],
        E_SHAPE: [(1, -1), (4, -1), (5, 0), (9, -1), (10, 0), (10, 33)],
        E_ALIGN: [(0, 8), (2, 8), (6, 2), (7, 2), (8, 2), (11, 8), (12, 2)]})


def test_quantize_checks(lib):
    qt = lambda *a: ctypes.byref(rfq._QT(*a))  # noqa: E731
    ok = (0, 1, 24, 128, 16, 16)
    good = [16, 128, 3, 16, 8, 16, qt(*ok), qt(*ok), None]
    _checks(lib.rfq_moe_quantize, good, {
        E_ARG: [(0, None), (3, None), (6, None), (6, qt(9, 1, 24, 128, 16, 16)), (6, qt(0, 1, 24, 128, None, 16))],
        E_SHAPE: [(1, -8), (2, -1), (4, 0), (4, 33), (6, qt(0, 1, 24, 96, 16, 16)), (7, qt(0, 1, 25, 128, 16, 16)),
                  (7, qt(0, 1, 24, 256, 16, 16))],
        E_ALIGN: [(0, 8), (1, 132), (3, 2), (5, 2), (6, qt(0, 1, 24, 128, 8, 16)), (7, qt(0, 1, 24, 128, 16, 8))],
        E_UNSUPPORTED: [(6, qt(3, 1, 24, 128, 16, 16)), (6, qt(0, 0, 24, 128, 16, 16)), (7, qt(3, 1, 24, 128, 16, 16)),
                        (7, qt(0, 0, 24, 128, 16, 16)), (6, qt(1, 1, 24, 128, 16, 16))]})


def test_binding_refuses(lib):
    f32, i32, b16 = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 8, dtype=torch.bfloat16)
    pair = torch.zeros(8, dtype=torch.int32)
    ws = torch.zeros(64, dtype=torch.int32)
    w = torch.zeros(4, 2)
    bad = [lambda: rfq.rfq_norm(f32, b16), lambda: rfq.rfq_norm(f32, torch.zeros(4, 9)), lambda: rfq.rfq_norm(f32, f32, weight=torch.zeros(7)),
           lambda: rfq.rfq_norm(f32, f32, weight=torch.zeros(8), bias=torch.zeros(8, dtype=torch.bfloat16)),
           lambda: rfq.rfq_norm(f32.t(), f32.t()), lambda: rfq.rfq_norm(f32, f32, mean=torch.zeros(3)), lambda: rfq.rfq_norm(f32.half(), f32.half()),
           lambda: rfq.rfq_norm_grad(f32, f32, torch.zeros(3), f32), lambda: rfq.rfq_norm_grad(f32, b16, torch.zeros(4), f32),
           lambda: rfq.rfq_norm_grad(f32, f32, torch.zeros(4), f32, dweight=torch.zeros(8)),
           lambda: rfq.rfq_norm_grad(f32, f32, torch.zeros(4), f32, dweight=torch.zeros(8).half(), workspace=f32),
           lambda: rfq.rfq_route(f32, i32, w.double()), lambda: rfq.rfq_route(f32, i32.long(), w), lambda: rfq.rfq_route(f32, i32[:3], w),
           lambda: rfq.rfq_route(torch.zeros(8, 4).t(), i32, w),
           lambda: rfq.rfq_route_grad(f32, i32, w, b16), lambda: rfq.rfq_route_grad(f32, i32, w[:3], f32),
           lambda: rfq.rfq_moe_sort(i32, pair, i32[:3], pair, ws), lambda: rfq.rfq_moe_sort(i32.long(), pair, i32, pair, ws),
           lambda: rfq.rfq_moe_sort(i32, pair, i32, pair, ws[:32]), lambda: rfq.rfq_moe_rows(-1, 1, 1),
           lambda: rfq.rfq_moe_gather(f32, i32, b16), lambda: rfq.rfq_moe_gather(f32, i32[:3], f32), lambda: rfq.rfq_moe_gather(f32, i32, torch.zeros(8, 9)),
           lambda: rfq.rfq_moe_gather(f32, i32, torch.zeros(9, 8), pair_of=pair),
           lambda: rfq.rfq_moe_combine(f32, i32, b16), lambda: rfq.rfq_moe_combine(f32, i32, f32, weights=w.double()),
           lambda: rfq.rfq_moe_combine(torch.zeros(8, 8)[::2], i32, f32),
           lambda: rfq.rfq_moe_combine_grad(f32, f32, i32, w, torch.zeros(5, 8), w), lambda: rfq.rfq_moe_combine_grad(f32, f32, i32, w, f32, w[:3]),
           lambda: rfq.rfq_moe_quantize(f32, i32, rfq.QTensor(0, 1, 8, 8, f32, f32)),
           lambda: rfq.rfq_moe_quantize(b16, i32, rfq.QTensor(0, 1, 8, 16, f32, f32)),
           lambda: rfq.rfq_moe_quantize(torch.zeros(4, 128, dtype=torch.bfloat16), i32, rfq.QTensor(0, 1, 8, 128, f32, torch.zeros(128))),
           lambda: rfq.rfq_moe_quantize(torch.zeros(4, 128, dtype=torch.bfloat16), i32, rfq.QTensor(0, 1, 8, 128, torch.zeros(128), f32))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    # tensors in host memory
    for f in (lambda: rfq.rfq_norm(f32, f32), lambda: rfq.rfq_route(f32, i32, w), lambda: rfq.rfq_moe_sort(i32, pair, i32, pair, ws),
              lambda: rfq.rfq_moe_gather(f32, i32, torch.zeros(8, 8)), lambda: rfq.rfq_moe_combine(f32, i32, f32)):
        with pytest.raises(ValueError, match="CUDA device"):
            f()


def test_launch_shapes(fake):
    """Every size that is taken gives a launch: threads and shared memory within
    the limits, on devices of different sizes."""
    for device in (0, 1):
        fake.device(device)
        sms = 76 if device == 1 else 152
        for dim in (1, 2, 7, 8, 31, 64, 80, 120, 128, 256, 264, 512, 1000, 1023, 1024, 2048, 4096, 4100, 5120, 5128, 8192, 8200, 8201, 8288, 9216, 10001, 11264, 12288, 12296, 13824, 16383, 16384):
            for dtype in (0, 1):
                for rows in (1, 5, 32760):
                    before = len(fake.launches())
                    assert fake.lib.rfq_norm(256, dim, dim, 256, dim, dim, dtype, rows, 1, dim, 0, 1e-6, 256, 256, 0, 256, 256, None) == rfq.RFQ_OK
                    assert fake.lib.rfq_norm_grad(256, dim, dim, 256, dim, dim, 256, dim, dim, dtype, rows, 1, dim, 0, 256, 256, 256, 0, 256, 256,
                                                  256, None) == rfq.RFQ_OK
                    for x, y, z, threads, cluster, smem in fake.launches()[before:]:
                        assert 1 <= threads <= 1024 and threads % 32 == 0 and x >= 1 and y == z == 1
                    x, _, _, threads, _, _ = fake.launches()[before + 1]
                    assert x * 2 * dim * 4 <= fake.lib.rfq_norm_grad_workspace_bytes(dim) <= 16 * sms * 2 * dim * 4
        # no rows: the sums of nothing are written, by one launch
        before = len(fake.launches())
        assert fake.lib.rfq_norm_grad(None, 8, 8, None, 8, 8, None, 8, 8, 1, 0, 1, 8, 0, None, None, 256, 0, 256, 256, 256, None) == rfq.RFQ_OK
        assert len(fake.launches()) == before + 1
        # the largest sizes of the calls that move rows
        most = 2 ** 31 // 8 - 1
        for dim, dtype in ((65536, 1), (65535, 1), (65535, 0), (1, 0)):
            assert fake.lib.rfq_moe_gather(256, dim, dtype, most, dim, 256, 8, 256, 256, 2 ** 31 - 1, None) == rfq.RFQ_OK
            assert fake.lib.rfq_moe_combine(256, dtype, 2 ** 31 - 1, dim, 256, 256, most, 8, 256, dim, None) == rfq.RFQ_OK
            assert fake.lib.rfq_moe_combine_grad(256, dim, 256, dtype, 2 ** 31 - 1, dim, 256, 256, 256, most, 8, 256, 256, None) == rfq.RFQ_OK
        q = ctypes.byref(rfq._QT(0, 1, 2 ** 31 - 1, 65536, 256, 256))
        assert fake.lib.rfq_moe_quantize(256, 65536, most, 256, 8, 256, q, q, None) == rfq.RFQ_OK
        for x, y, z, threads, cluster, smem in fake.launches()[before:]:
            assert 1 <= x < 2 ** 31 and 1 <= y <= 65535 and z == 1 and threads <= 1024
        for tokens in (0, 1, 512, 513, 4096, 262144, 2 ** 31 // 8 - 2 ** 13):
            before = len(fake.launches())
            assert fake.lib.rfq_moe_sort(256, tokens, 8, 128, 128, 256, 256, 256, 2 ** 31 - 1, 256, None) == rfq.RFQ_OK
            (x, _, _, threads, cluster, _), = fake.launches()[before:]
            assert threads in (256, 512, 1024) and x == cluster <= 8


def test_references_against_autograd():
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    for rms in (False, True):
        x, w, b, dy = rnd(5, 3, 17).requires_grad_(), rnd(17).requires_grad_(), rnd(17).requires_grad_(), rnd(5, 3, 17)
        y, m, r = moe_ref.norm(x, w, b, 1e-6, rms)
        y.backward(dy)
        dx, dw, db = moe_ref.norm_grad(dy, x.detach(), m.detach(), r.detach(), w.detach(), rms)
        for a, c in ((dx, x.grad), (dw, w.grad), (db, b.grad)):
            torch.testing.assert_close(a, c)
    for normalize in (False, True):
        l, dw = rnd(6, 9).requires_grad_(), rnd(6, 4)
        ids, wt = moe_ref.route(l.detach(), 4, normalize)
        p = torch.softmax(l, -1).gather(1, ids.long())
        p = p / p.sum(-1, keepdim=True) if normalize else p
        torch.testing.assert_close(p.detach(), wt)
        p.backward(dw)
        torch.testing.assert_close(moe_ref.route_grad(l.detach(), ids, dw, normalize)[0], l.grad)
