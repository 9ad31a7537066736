"""What the header says of the entry points around a mixture-of-experts block,
in calls that lie at the edge of it."""
import pytest
import torch

from gpu_util import DEV
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [256, 257, 5120])
def test_rows_with_inf_and_nan(dim, dtype):
    """By the formula: a NaN, or an Inf in a layer norm, makes a row NaN; in an
    RMS norm an Inf gives rstd = 0, NaN in its place and the bias in the others."""
    g = torch.Generator().manual_seed(dim)
    x = torch.randn(6, dim, generator=g).to(dtype)
    x[1, 7], x[2, dim - 1], x[4, 0] = float("inf"), float("-inf"), float("nan")
    x[2, 3] = float("inf")
    b = torch.randn(dim, generator=g)
    for kind in (rfq.RFQ_NORM_LAYER, rfq.RFQ_NORM_RMS):
        y, clean = torch.empty(6, dim, dtype=dtype, device=DEV), torch.empty(6, dim, dtype=dtype, device=DEV)
        rstd = torch.empty(6, device=DEV)
        rfq.rfq_norm(x.to(DEV), y, bias=b.to(DEV), kind=kind, rstd=rstd)
        rfq.rfq_norm(torch.where(x.isfinite(), x, 0).to(DEV), clean, bias=b.to(DEV), kind=kind)
        y, rstd = y.cpu(), rstd.cpu()
        assert torch.equal(y[[0, 3, 5]], clean.cpu()[[0, 3, 5]]) and y[4].isnan().all() and rstd[4].isnan()
        for r in (1, 2):
            inf = x[r].isinf()
            if kind == rfq.RFQ_NORM_LAYER:
                assert y[r].isnan().all()
            else:
                assert rstd[r] == 0 and y[r][inf].isnan().all() and torch.equal(y[r][~inf], b.to(dtype)[~inf])
