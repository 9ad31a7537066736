"""The example layer (examples/decode_layer.py) against the same layer in 64
bits: prompts of several lengths, then single tokens, then a prompt long
enough for the RFQ linear layer."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import serving_ref as ref
from conftest import ROOT
from gpu_util import DEV, qtensor_host
from paper_2608_26581_gb300 import rfq
from paper_2608_26581_gb300.synth import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location("decode_layer", os.path.join(ROOT, "examples", "decode_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _bf16(a):
    return bf16_bits_to_f32(f32_to_bf16_bits(np.asarray(a, np.float32))).astype(np.float64)


@pytest.mark.parametrize("fmt", [rfq.RFQ_FMT_MXFP4, rfq.RFQ_FMT_HIF4])
def test_layer_against_64_bits(orc, fmt):
    R, hidden, H, KV, D = 3, 256, 8, 2, 64
    layer = _example().AttentionLayer(R, 120, hidden=hidden, heads=H, kv_heads=KV, head_dim=D, page_size=16, fmt=fmt, sections=(12, 10, 10))
    ofmt = orc.FMT_HIF4 if fmt == rfq.RFQ_FMT_HIF4 else orc.FMT_MXFP4
    w = []
    for q in (layer.w_qkv, layer.w_out):
        w.append(orc.dequant(ofmt, *qtensor_host(q), q.rows, q.k))
    freq, axis = layer.inv_freq.double().cpu().numpy(), layer.axis_of.cpu().numpy()
    keys, values = [np.zeros((0, KV, D))] * R, [np.zeros((0, KV, D))] * R
    rng = np.random.default_rng(0)
    # (added, image grid?): short prompts, single tokens, one more chunk, a long prompt (more than 32 tokens)
    for added, grid in (([5, 17, 1], False), ([1, 1, 1], False), ([1, 1, 1], True), ([0, 3, 9], True), ([40, 2, 0], False)):
        T = sum(added)
        xb = f32_to_bf16_bits(rng.standard_normal((T, hidden)).astype(np.float32))
        gr = rng.integers(0, 9, (3, T)).astype(np.int32) if grid else None
        b = layer.buffers(T)
        y = layer.step(torch.from_numpy(xb.view(np.int16)).to(DEV).view(torch.bfloat16), torch.tensor(added, dtype=torch.int32, device=DEV), b,
                       None if gr is None else torch.from_numpy(gr).to(DEV), single=added == [1] * R)
        layer.check()
        x = bf16_bits_to_f32(xb).astype(np.float64)
        if T > 32:      # the RFQ linear layer: x as its two quantized terms
            d = orc.quantize_act(xb, ofmt)
            x = orc.dequant(ofmt, d["main_codes"], d["main_scales"], T, hidden) + orc.dequant(ofmt, d["res_codes"], d["res_scales"], T, hidden)
        qkv = _bf16(x @ w[0].T).reshape(T, H + 2 * KV, D)
        start = np.concatenate([[0], np.cumsum(added)])
        pos = np.concatenate([len(keys[r]) + np.arange(added[r]) for r in range(R)]).astype(np.int32)
        pos = np.stack([pos] * 3) + (0 if gr is None else gr)
        qk = _bf16(ref.rope(qkv[:, :H + KV], pos, freq, axis, False, False))
        for r in range(R):
            s = slice(start[r], start[r + 1])
            for store, rows in ((keys, qk[s, H:]), (values, qkv[s, H + KV:])):
                n = rows.shape[0] * KV
                if n:
                    val = orc.dequant(ofmt, *orc.quantize(ofmt, rows.reshape(n, D)), n, D).reshape(-1, KV, D)
                    store[r] = np.concatenate([store[r], val])
        o, _ = ref.attention(qk[:, :H], keys, values, start, [len(k) for k in keys], D ** -0.5, 0)
        o = _bf16(o)
        if T > 32:
            d = orc.quantize_act(f32_to_bf16_bits(o.reshape(T, -1).astype(np.float32)), ofmt)
            o = orc.dequant(ofmt, d["main_codes"], d["main_scales"], T, H * D) + orc.dequant(ofmt, d["res_codes"], d["res_scales"], T, H * D)
        want = o.reshape(T, -1) @ w[1].T
        got = y.double().cpu().numpy()
        assert layer.lengths.tolist() == [len(k) for k in keys]
        # bf16 roundings that fall on the other side (2^-8 each) move a 4-bit
        # code of a key or value by a step now and then: a few percent of it in
        # few places; an error of the layer's logic is of order one
        assert np.linalg.norm(got - want) <= 0.03 * np.linalg.norm(want)
