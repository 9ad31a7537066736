"""Kernels of the serving calls may start before the kernel in front of them
has finished: a step's calls in a row, each reading what the one before wrote,
give the same bits as with a wait between them, also from a CUDA graph."""
import pytest
import torch

from gpu_util import DEV
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu


def _step(wait, rounds=20, graph=False):
    """Slots -> projection -> rotary -> append -> attention -> projection, the
    output fed back in; returns the last output and the cache's bytes."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    R, H, KV, D, K, page = 7, 8, 2, 64, 512, 16
    F, L = rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA
    w = [rfq.empty_qtensor(F, L, n, k) for n, k in (((H + 2 * KV) * D, K), (K, H * D))]
    for q in w:
        rfq.rfq_quantize_weight((torch.randn(q.k, q.rows, generator=g, device=DEV) * 0.05).bfloat16(), q)
    cache = rfq.empty_kv_cache(F, KV, D, page, 64)
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.zero_()
    i32 = dict(dtype=torch.int32, device=DEV)
    cached, added, table = torch.zeros(R, **i32), torch.ones(R, **i32), torch.zeros(R, 8, **i32)
    free, count = torch.arange(64, **i32), torch.full((1,), 64, **i32)
    start, slots, pos = torch.zeros(R + 1, **i32), torch.zeros(R, dtype=torch.int64, device=DEV), torch.zeros(1, R, **i32)
    ws, wa = torch.zeros(64, **i32), rfq.kv_attention_workspace(H, D)
    freq, axis = 1e4 ** (-torch.arange(D // 2, device=DEV) / (D // 2)), torch.zeros(D // 2, **i32)
    x = torch.randn(R, K, generator=g, device=DEV).bfloat16()
    qkv = torch.empty(R, H + 2 * KV, D, dtype=torch.bfloat16, device=DEV)
    o = torch.empty(R, H, D, dtype=torch.bfloat16, device=DEV)
    pause = torch.cuda.synchronize if wait else lambda: None

    def once():
        rfq.rfq_slot_map(cached, added, page, table, free, count, count, cached, start, slots, pos[0], ws)
        pause()
        rfq.rfq_matvec(x, w[0], qkv.view(R, -1))
        pause()
        rfq.rfq_rope(qkv[:, :H + KV], qkv[:, :H + KV], pos, freq, axis)
        pause()
        rfq.rfq_kv_append(qkv[:, H:H + KV], qkv[:, H + KV:], slots, cache)
        pause()
        rfq.rfq_kv_attention(qkv[:, :H], cache, table, cached, o, wa)
        pause()
        rfq.rfq_matvec(o.view(R, -1), w[1], x)
        pause()
    if graph:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            once()
        for _ in range(rounds):
            gr.replay()
    else:
        for _ in range(rounds):
            once()
    torch.cuda.synchronize()
    assert rfq.rfq_workspace_status(ws) == rfq.RFQ_OK and rfq.rfq_workspace_status(wa) == rfq.RFQ_OK
    return x.clone(), cached.clone(), cache.k_codes.clone(), cache.v_codes.clone(), cache.k_scales.clone()


def test_back_to_back_equals_with_waits():
    want = _step(wait=True)
    assert torch.isfinite(want[0].float()).all() and int(want[1][0]) == 20
    for graph in (False, True):
        for _ in range(3):
            got = _step(wait=False, graph=graph)
            for a, b in zip(got, want):
                assert torch.equal(a, b)
