"""What the header says of the entry points around a mixture-of-experts block,
in calls that lie at the edge of it."""
import pytest
import torch

import moe_ref
from gpu_util import DEV, guarded_full
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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [33, 1000, 2048])
def test_rows_that_two_pairs_name(dim, dtype):
    """Each element is one of the two's, and every dweight is right."""
    g = torch.Generator().manual_seed(dim)
    x, y, w = torch.randn(40, dim, generator=g).to(dtype), torch.randn(20, dim, generator=g).to(dtype), torch.randn(40, 1, generator=g)
    row_of = (torch.arange(40) % 20)[:, None].int()
    out = guarded_full((20, dim), float("nan"), dtype)
    rfq.rfq_moe_gather(x.to(DEV), row_of.to(DEV), out)
    assert ((out.cpu() == x[:20]) | (out.cpu() == x[20:])).all()
    dy, dw = guarded_full((20, dim), float("nan"), dtype), guarded_full((40, 1), float("nan"), F32)
    rfq.rfq_moe_combine_grad(x.to(DEV), y.to(DEV), row_of.to(DEV), w.to(DEV), dy, dw)
    each = (x.float() * w).to(dtype)                   # one product of fp32, rounded
    assert ((dy.cpu() == each[:20]) | (dy.cpu() == each[20:])).all()
    dots = x.double() * y.double().repeat(2, 1)
    # a lane's own products and additions, then five over lanes
    e = (2 * -(-dim // 32) + 8) * moe_ref.U * dots.abs().sum(-1)
    assert ((dw.double().cpu()[:, 0] - dots.sum(-1)).abs() <= e).all()
