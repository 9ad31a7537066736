"""rfq_matvec against the product in 64 bits of the oracle's dequantized W~."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, guarded_full, to_dev_bf16
from paper_2608_26581_gb300 import rfq
from paper_2608_26581_gb300.synth import bf16_bits_to_f32, f32_to_bf16_bits, make_weight

pytestmark = pytest.mark.gpu
MX, HI, ROW, MMA = rfq.RFQ_FMT_MXFP4, rfq.RFQ_FMT_HIF4, rfq.RFQ_SCALE_ROWMAJOR, rfq.RFQ_SCALE_MMA


def _values(orc, wb, fmt):
    K, N = wb.shape
    codes, scales = orc.quantize_weight(wb, fmt)
    return orc.dequant(fmt, codes, scales, N, K)


def _run(xd, wq, M, N, dtype):
    y = guarded_full((M, N), 7.0, dtype)
    rfq.rfq_matvec(xd, wq, y)
    return y


def check(y, x, w, dtype):
    """x in f16 is exact but for 2^-39 of a stretch's maximum; products are
    exact in fp32 and their sums off by 2^-24 a step of at most K / 4 steps
    and the joins: 2^-24 (K / 4 + 64) of sum |x w| is never reached; its
    square root growth stays below 2^-18.  bf16: plus half an ulp, 2^-8."""
    want = x @ w.T
    mag = np.abs(x) @ np.abs(w).T
    bound = 2.0 ** -18 * mag + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0) + 1e-35
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= bound).all(), f"worst {np.max(err / bound):.3f} of the bound"


@pytest.mark.parametrize("fmt,layout", [(MX, ROW), (MX, MMA), (HI, ROW), (HI, MMA)])
@pytest.mark.parametrize("M,K,N", [(1, 128, 16), (1, 4096, 300), (3, 1152, 65), (8, 2048, 128), (9, 640, 513), (16, 3200, 64),
                                   (17, 384, 1), (32, 5120, 200), (2, 12288, 130), (5, 8320, 640)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matches_the_product(orc, fmt, layout, M, K, N, dtype):
    rng = np.random.default_rng(K + N)
    xb = f32_to_bf16_bits((rng.standard_normal((M, K)) * np.where(rng.random(K) < 0.02, 50, 1)).astype(np.float32))
    wb = make_weight(K, N, seed=K)
    wq = rfq.empty_qtensor(fmt, layout, N, K)
    rfq.rfq_quantize_weight(to_dev_bf16(wb), wq)
    y = _run(to_dev_bf16(xb), wq, M, N, dtype)
    check(y, bf16_bits_to_f32(xb).astype(np.float64), _values(orc, wb, orc.FMT_HIF4 if fmt == HI else orc.FMT_MXFP4), dtype)


@pytest.mark.parametrize("fmt,K", [(MX, 32), (MX, 96), (MX, 1120), (MX, 2080), (HI, 64), (HI, 192), (HI, 1088)])
def test_odd_k_row_major_scales(orc, fmt, K):
    rng = np.random.default_rng(K)
    M, N = 4, 77
    xb, wb = f32_to_bf16_bits(rng.standard_normal((M, K)).astype(np.float32)), make_weight(K, N, seed=3)
    wq = rfq.empty_qtensor(fmt, ROW, N, K)
    rfq.rfq_quantize_weight(to_dev_bf16(wb), wq)
    y = _run(to_dev_bf16(xb), wq, M, N, torch.float32)
    check(y, bf16_bits_to_f32(xb).astype(np.float64), _values(orc, wb, orc.FMT_HIF4 if fmt == HI else orc.FMT_MXFP4), torch.float32)


@pytest.mark.parametrize("fmt", [MX, HI])
def test_wide_ranges_and_strided_rows(orc, fmt):
    """Rows of x far apart in magnitude, a massive element, zeros; weights whose
    block scales span 2^60; rows of x inside a wider tensor."""
    rng = np.random.default_rng(1)
    M, K, N = 6, 1024, 96
    x = rng.standard_normal((M, K)) * (2.0 ** np.array([-100, -20, 0, 0, 30, 90]))[:, None]
    x[2] = 0
    x[3, 17] *= 5000
    w = rng.standard_normal((K, N)) * 2.0 ** rng.integers(-30, 30 if fmt == MX else 6, (K // 32, 1)).repeat(32, 0)
    if fmt == HI:
        w = rng.standard_normal((K, N)) * 2.0 ** rng.integers(-30, 6, (K // 64, 1)).repeat(64, 0)
    xb, wb = f32_to_bf16_bits(x.astype(np.float32)), f32_to_bf16_bits(w.astype(np.float32))
    wq = rfq.empty_qtensor(fmt, MMA, N, K)
    rfq.rfq_quantize_weight(to_dev_bf16(wb), wq)
    wide = torch.full((M, K + 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 32:32 + K] = to_dev_bf16(xb)
    y = _run(wide[:, 32:32 + K], wq, M, N, torch.float32)
    check(y, bf16_bits_to_f32(xb).astype(np.float64), _values(orc, wb, orc.FMT_HIF4 if fmt == HI else orc.FMT_MXFP4), torch.float32)


def test_same_bits_twice(orc):
    wb = make_weight(4096, 1000, seed=2)
    wq = rfq.empty_qtensor(MX, MMA, 1000, 4096)
    rfq.rfq_quantize_weight(to_dev_bf16(wb), wq)
    x = torch.randn(7, 4096, device=DEV).bfloat16()
    a = _run(x, wq, 7, 1000, torch.float32)
    for _ in range(3):
        assert torch.equal(a, _run(x, wq, 7, 1000, torch.float32))


def test_nothing_to_do_and_refusals():
    wq = rfq.empty_qtensor(MX, MMA, 64, 128)
    rfq.rfq_matvec(torch.empty(0, 128, dtype=torch.bfloat16, device=DEV), wq, torch.empty(0, 64, device=DEV))
    x, y = torch.zeros(2, 128, dtype=torch.bfloat16, device=DEV), torch.empty(2, 64, device=DEV)
    for bad in ((x.float(), wq, y), (x, wq, y.half()), (x[:, :64], wq, y), (x, wq, y[:, :32])):
        with pytest.raises(ValueError):
            rfq.rfq_matvec(*bad)
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_matvec(torch.zeros(33, 128, dtype=torch.bfloat16, device=DEV), wq, torch.empty(33, 64, device=DEV))
    assert e.value.status == rfq.RFQ_ERR_SHAPE
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_matvec(x, rfq.empty_qtensor(rfq.RFQ_FMT_MXFP8, MMA, 64, 128), y)
    assert e.value.status == rfq.RFQ_ERR_UNSUPPORTED
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_matvec(torch.zeros(2, 132, dtype=torch.bfloat16, device=DEV)[:, :128], wq, y)
    assert e.value.status == rfq.RFQ_ERR_ALIGNMENT
