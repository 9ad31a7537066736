"""What the header says of the entry points around a mixture-of-experts block,
without a GPU: sizes that are taken and refused, launches of unusual calls."""
import pytest

from fake_cuda import FakeCuda
from paper_2608_26581_gb300 import rfq


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeCuda(tmp_path_factory.mktemp("fake"))


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
