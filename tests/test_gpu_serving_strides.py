"""Strides of axes that have one element: tensors carry any number there, and the
serving calls do not look at it."""
import pytest
import torch

from gpu_util import DEV
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu


def _odd(x, *axes):
    """The same values with a stride of one element along `axes`, which have one element."""
    strides = [1 if i in axes else s for i, s in enumerate(x.stride())]
    return x.as_strided(x.shape, strides)


@pytest.mark.parametrize("fmt", [rfq.RFQ_FMT_MXFP4, rfq.RFQ_FMT_HIF4])
def test_one_row_of_a_product(fmt):
    w = rfq.empty_qtensor(fmt, rfq.RFQ_SCALE_MMA, 70, 256)
    rfq.rfq_quantize_weight(torch.randn(256, 70, device=DEV).bfloat16(), w)
    column = torch.randn(256, 1, device=DEV).bfloat16()
    y, want = torch.empty(1, 70, device=DEV), torch.empty(1, 70, device=DEV)
    rfq.rfq_matvec(column.t().clone(memory_format=torch.contiguous_format).view(1, 256), w, want)
    assert column.t().stride() == (1, 1)
    rfq.rfq_matvec(column.t(), w, y)
    assert torch.equal(y, want)


@pytest.mark.parametrize("T,H", [(1, 1), (1, 2), (5, 1)])
def test_one_token_or_head(T, H):
    D, page = 64, 16
    axes = [i for i, n in enumerate((T, H)) if n == 1]
    k, v, q = (torch.randn(T, H, D, device=DEV).bfloat16() for _ in range(3))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    pos, freq, axis = i32([list(range(T))]), torch.rand(D // 2, device=DEV), i32([0] * (D // 2))
    turned = [torch.empty_like(k) for _ in range(2)]
    rfq.rfq_rope(k, turned[0], pos, freq, axis)
    rfq.rfq_rope(_odd(k, *axes), _odd(turned[1], *axes), pos, freq, axis)
    assert torch.equal(*turned)
    got = []
    for x in (lambda t: t, lambda t: _odd(t, *axes)):
        cache = rfq.empty_kv_cache(rfq.RFQ_FMT_MXFP4, H, D, page, 1)
        for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
            t.zero_()
        rfq.rfq_kv_append(x(k), x(v), torch.arange(T, device=DEV), cache)
        out = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
        rfq.rfq_kv_attention(x(q), cache, i32([[0]]), i32([T]), out, rfq.kv_attention_workspace(H, D), q_start=i32([0, T]))
        got.append((cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, out))
    for a, b in zip(*got):
        assert torch.equal(a, b)
