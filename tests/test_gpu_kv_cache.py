"""The paged 4-bit cache: bytes of rfq_kv_append equal the oracle's codes and
scales at their documented places, and rfq_kv_read gives their values back."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import CANARY, DEV, guarded_bytes, guarded_full
from paper_2608_26581_gb300 import rfq
from paper_2608_26581_gb300.synth import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def new_cache(fmt, heads, D, page, pages, fill=0x5A):
    cb, sb = rfq.rfq_kv_cache_bytes(fmt, heads, D, page, pages)
    a = [guarded_bytes(n) for n in (cb, sb, cb, sb)]
    for t in a:
        t.fill_(fill)
    return rfq.KVCache(fmt, heads, D, page, pages, *a)


def bits_to_dev(bits):
    return torch.from_numpy(bits.view(np.int16)).to(DEV).view(torch.bfloat16)


def draw_kv(T, H, D, seed, wide=False):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, H, D)) * np.where(rng.random((H, D)) < 0.05, 40, 1)
    if wide:
        x *= 2.0 ** rng.integers(-130, 120, (T, H, 1))
        x[0] = 0
        x[-1, :, ::3] = -0.0
    return f32_to_bf16_bits(x.astype(np.float32))


@pytest.mark.parametrize("fmt", [ref.FMT_MXFP4, ref.FMT_HIF4])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,H,page,pages", [(1, 1, 16, 1), (3, 8, 16, 9), (61, 3, 48, 4), (200, 2, 64, 5)])
def test_append_and_read(orc, fmt, D, T, H, page, pages):
    rng = np.random.default_rng(T + D)
    kb, vb = draw_kv(T, H, D, 1, wide=True), draw_kv(T, H, D, 2)
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    if T > 2:
        slots[1], slots[2] = -1, pages * page       # tokens without a slot
    cache = new_cache(fmt, H, D, page, pages)
    # keys and values of one packed projection: [T][2 H + 1][D]
    packed = torch.zeros(T, 2 * H + 1, D, dtype=torch.bfloat16, device=DEV)
    packed[:, :H], packed[:, H + 1:] = bits_to_dev(kb), bits_to_dev(vb)
    s = torch.from_numpy(slots).to(DEV)
    rfq.rfq_kv_append(packed[:, :H], packed[:, H + 1:], s, cache)
    outs = {}
    for dt in (torch.float32, torch.bfloat16):
        k, v = guarded_full((T, H, D), 7.0, dt), guarded_full((T, H, D), 7.0, dt)
        rfq.rfq_kv_read(cache, s, k, v)
        outs[dt] = (k, v)
    ofmt = orc.FMT_HIF4 if fmt == ref.FMT_HIF4 else orc.FMT_MXFP4
    for x, which in ((kb, 0), (vb, 1)):
        rows = bf16_bits_to_f32(x).astype(np.float64).reshape(T * H, D)
        codes, scales = orc.quantize(ofmt, rows)
        kc, vc, sc = ref.cache_bytes(codes.reshape(T, H, -1), scales.reshape(T, H, -1), fmt, D, page, pages, H, slots)
        for arr, want in ((cache.v_codes if which else cache.k_codes, vc if which else kc),
                          (cache.v_scales if which else cache.k_scales, sc)):
            exp = np.full(arr.numel(), 0x5A, np.uint8)
            exp[list(want.keys())] = list(want.values())
            np.testing.assert_array_equal(arr.cpu().numpy(), exp)
        val = orc.dequant(ofmt, codes, scales, T * H, D).reshape(T, H, D)
        val[(slots < 0) | (slots >= pages * page)] = 0
        np.testing.assert_array_equal(outs[torch.float32][which].double().cpu().numpy(), val.astype(np.float32))
        b16 = bf16_bits_to_f32(f32_to_bf16_bits(val.astype(np.float32)))
        np.testing.assert_array_equal(outs[torch.bfloat16][which].float().cpu().numpy(), b16)


def test_append_many_tokens(orc):
    """More tokens than the grid has lanes at once: values against the oracle."""
    T, H, D, page, pages = 9000, 8, 128, 64, 150
    kb, vb = draw_kv(T, H, D, 5), draw_kv(T, H, D, 6)
    cache = new_cache(ref.FMT_MXFP4, H, D, page, pages)
    s = torch.randperm(pages * page)[:T].to(DEV)
    rfq.rfq_kv_append(bits_to_dev(kb), bits_to_dev(vb), s, cache)
    k, v = guarded_full((T, H, D), 7.0, torch.float32), guarded_full((T, H, D), 7.0, torch.float32)
    rfq.rfq_kv_read(cache, s, k, v)
    for x, got in ((kb, k), (vb, v)):
        rows = bf16_bits_to_f32(x).astype(np.float64).reshape(T * H, D)
        val = orc.dequant(orc.FMT_MXFP4, *orc.quantize(orc.FMT_MXFP4, rows), T * H, D)
        np.testing.assert_array_equal(got.double().cpu().numpy().reshape(T * H, D), val)


def test_zero_tokens_and_refusals():
    cache = new_cache(ref.FMT_MXFP4, 2, 64, 16, 3)
    z = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    rfq.rfq_kv_append(z, z, none, cache)
    rfq.rfq_kv_read(cache, none, z, z)
    x, s = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV)
    for bad in ((x.float(), x.float(), s, cache), (x, x, s.int(), cache), (x[:, :1], x[:, :1], s, cache), (x, x, s[:1], cache)):
        with pytest.raises(ValueError):
            rfq.rfq_kv_append(*bad)
    odd = torch.zeros(2, 2, 66, dtype=torch.bfloat16, device=DEV)[:, :, :64]
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_kv_append(odd, odd, s, cache)
    assert e.value.status == rfq.RFQ_ERR_ALIGNMENT
    assert (cache.k_codes == 0x5A).all() and CANARY
