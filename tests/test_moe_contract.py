"""What the header says of the entry points around a mixture-of-experts block,
without a GPU: sizes that are taken and refused, launches of unusual calls."""
import ctypes

import pytest

from fake_kernels import FakeKernels
from paper_2608_26581_gb300 import rfq


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeKernels(tmp_path_factory.mktemp("fake"))


def test_rows_only_where_the_sort_takes_the_sizes(fake):
    """rfq_moe_rows: -1 exactly where rfq_moe_sort gives RFQ_ERR_SHAPE, else rows
    that fit 31 bits."""
    most = 2 ** 31 - 1
    for top_k, experts, align in ((8, 256, 4096), (1, 1, 1), (1, 256, 4096), (32, 256, 128), (8, 128, 1), (3, 5, 7)):
        border = (most - experts * align) // top_k
        for tokens in (0, 1, border - 1, border, border + 1, most // top_k, most // top_k + 1):
            rows = fake.lib.rfq_moe_rows(tokens, top_k, experts, align)
            status = fake.lib.rfq_moe_sort(256, tokens, top_k, experts, align, 256, 256, 256, max(rows, 0), 256, None)
            assert status == (rfq.RFQ_ERR_SHAPE if rows < 0 else rfq.RFQ_OK), (tokens, top_k, experts, align)
            assert rows <= most and (rows >= 0) == (tokens <= border)


def test_strides_along_one_element(fake):
    """A stride between tokens where there is one token, or between heads where
    there is one head, changes nothing: the same kernels, launched the same way."""
    qt = lambda: ctypes.byref(rfq._QT(0, 1, 24, 128, 256, 256))  # noqa: E731
    # (call, arguments with odd strides, which strides those are)
    norm = lambda t, h: (t, h, 256, t, h)  # noqa: E731
    cases = []
    for tokens, heads, odd in ((700, 1, (128, 131)), (1, 40, (5121, 128)), (1, 1, (129, 131)), (1, 1, (-1, -1))):
        for dtype in (0, 1):
            args = lambda t, h: (256, *norm(t, h), dtype, tokens, heads, 128, 0, 1e-6, 256, 256, 0, 256, 256, None)  # noqa: E731
            even = (odd[0] if tokens > 1 else 0, odd[1] if heads > 1 else 0)
            cases.append(("rfq_norm", args(*odd), args(*even)))
            args = lambda t, h: (256, *norm(t, h), 256, t, h, dtype, tokens, heads, 128, 0, 256, 256, 256, 0, 256, 256, 256, None)  # noqa: E731
            cases.append(("rfq_norm_grad", args(*odd), args(*even)))
    for dtype in (0, 1):
        for row in (129, -1):
            cases += [("rfq_route", *((256, r, dtype, 1, 128, 8, 1, 256, 256, None) for r in (row, 0))),
                      ("rfq_route_grad", *((256, r, dtype, 1, 128, 8, 1, 256, 256, 256, r, None) for r in (row, 0))),
                      ("rfq_moe_gather", *((256, r, dtype, 1, 128, 256, 8, 256, 256, 24, None) for r in (row, 0))),
                      ("rfq_moe_combine", *((256, dtype, 24, 128, 256, 256, 1, 8, 256, r, None) for r in (row, 0))),
                      ("rfq_moe_combine_grad", *((256, r, 256, dtype, 24, 128, 256, 256, 256, 1, 8, 256, 256, None) for r in (row, 0)))]
    cases += [("rfq_moe_quantize", *((256, r, 1, 256, 8, 256, qt(), qt(), None) for r in (row, 0))) for row in (129, -1)]
    for f, odd, even in cases:
        want = fake.call(f, *even)
        assert want[0] == rfq.RFQ_OK and want[1]
        assert fake.call(f, *odd) == want, (f, odd)
