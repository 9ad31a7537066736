"""One attention layer answering a batch of requests on a 4-bit cache.

Every step adds tokens to some requests (a prompt, or one token each) and runs

    slot map -> query/key/value projection -> rotary positions -> cache append
    -> attention over the cache -> output projection

with the weights and the cache in MXFP4 or HiF4.  Steps of up to 32 tokens
project with rfq_matvec (x in bf16), longer ones with the RFQ linear layer
(x quantized with its residual).  A step's sizes are fixed by its tensors, so a
decoding step can be captured in a CUDA graph and replayed while the requests
grow.

    python examples/decode_layer.py [--requests 16] [--prompt 200] [--steps 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_26581_gb300 import rfq  # noqa: E402


class AttentionLayer:
    """Weights, the paged cache and the bookkeeping of `requests` requests.
    The defaults are the attention of a Qwen3-VL-8B layer (hidden 4096, 32
    query heads, 8 key heads of 128); weights are random."""

    def __init__(self, requests, max_tokens, hidden=4096, heads=32, kv_heads=8, head_dim=128, page_size=64, fmt=rfq.RFQ_FMT_MXFP4,
                 sections=(24, 20, 20), base=5e6, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.hidden, self.heads, self.kv_heads, self.head_dim, self.page_size = hidden, heads, kv_heads, head_dim, page_size
        self.w_qkv = self._weight(hidden, (heads + 2 * kv_heads) * head_dim, fmt, g)
        self.w_out = self._weight(heads * head_dim, hidden, fmt, g)
        width = -(-max_tokens // page_size)
        pages = requests * width
        self.cache = rfq.empty_kv_cache(fmt, kv_heads, head_dim, page_size, pages)
        self.lengths = torch.zeros(requests, **i32)
        self.table = torch.zeros(requests, width, **i32)
        self.free, self.count = torch.arange(pages, **i32), torch.full((1,), pages, **i32)
        self.ws = torch.zeros(64, **i32)
        self.attn_ws = rfq.kv_attention_workspace(heads, head_dim)
        # one progression of frequencies, its pairs shared out to time, height and width
        pairs = head_dim // 2
        self.inv_freq = (base ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float()
        share = torch.tensor(sections, device="cuda") * pairs // sum(sections)
        share[0] += pairs - share.sum()
        self.axis_of = torch.repeat_interleave(torch.arange(3, device="cuda"), share).int()

    def _weight(self, k, n, fmt, g):
        w = (torch.randn(k, n, generator=g, device="cuda") * k ** -0.5).bfloat16()
        q = rfq.empty_qtensor(fmt, rfq.RFQ_SCALE_MMA, n, k)
        rfq.rfq_quantize_weight(w, q)
        return q

    def buffers(self, tokens):
        """The tensors of a step of `tokens` tokens, kept for as long as such steps are run."""
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        H, KV, D = self.heads, self.kv_heads, self.head_dim
        b = {"qkv": torch.empty(tokens, H + 2 * KV, D, **bf16), "o": torch.empty(tokens, H, D, **bf16),
             "y": torch.empty(tokens, self.hidden, **bf16), "slots": torch.empty(tokens, dtype=torch.int64, device="cuda"),
             "start": torch.empty(self.lengths.numel() + 1, dtype=torch.int32, device="cuda"),
             "pos": torch.zeros(3, tokens, dtype=torch.int32, device="cuda")}
        if tokens > 32:
            for name, w in (("x", self.w_qkv), ("a", self.w_out)):
                b[name] = [rfq.empty_qtensor(w.fmt, rfq.RFQ_SCALE_MMA, tokens, w.k) for _ in range(2)]
                if w.fmt == rfq.RFQ_FMT_HIF4:
                    b[name + "w"] = torch.empty(w.rows, w.k, **bf16)
                    rfq.rfq_dequant(w, b[name + "w"])
        return b

    def _project(self, x, w, y, b, name):
        if x.shape[0] <= 32:
            rfq.rfq_matvec(x, w, y)
            return
        xq, xr = b[name]
        rfq.rfq_quantize_act(x, xq, xr)
        wq = rfq.bf16_operand(b[name + "w"]) if w.fmt == rfq.RFQ_FMT_HIF4 else w
        rfq.rfq_linear(xq, xr, None, 256, wq, y, rfq.RFQ_OUT_BF16, self.ws)

    def step(self, x, added, b, grid=None, single=False):
        """x bf16 [tokens, hidden]: the step's tokens, request after request;
        added int32 [requests]: how many are each request's (all on the GPU).
        grid: int32 [3, tokens] added to the text positions (places in an image
        or a clip), or None.  single: every request adds one token.  Returns
        the layer's output, a tensor of b."""
        H, KV = self.heads, self.kv_heads
        pos = b["pos"]
        rfq.rfq_slot_map(self.lengths, added, self.page_size, self.table, self.free, self.count, self.count, self.lengths, b["start"],
                         b["slots"], pos[0], self.ws)
        self._project(x, self.w_qkv, b["qkv"].view(x.shape[0], -1), b, "x")
        pos[1:].copy_(pos[:1])
        if grid is not None:
            pos += grid
        turned = b["qkv"][:, :H + KV]
        rfq.rfq_rope(turned, turned, pos, self.inv_freq, self.axis_of, pairing=rfq.RFQ_ROPE_HALF)
        rfq.rfq_kv_append(b["qkv"][:, H:H + KV], b["qkv"][:, H + KV:], b["slots"], self.cache)
        rfq.rfq_kv_attention(b["qkv"][:, :H], self.cache, self.table, self.lengths, b["o"], self.attn_ws,
                             q_start=None if single else b["start"])
        self._project(b["o"].view(x.shape[0], -1), self.w_out, b["y"], b, "a")
        return b["y"]

    def check(self):
        """Raises if a step recorded a device status."""
        for w in (self.ws, self.attn_ws):
            s = rfq.rfq_workspace_status(w)
            if s != rfq.RFQ_OK:
                raise rfq.RFQError(s, "AttentionLayer")


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=200)
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args()
    R = a.requests
    layer = AttentionLayer(R, a.prompt + a.steps + 8)
    x = torch.randn(R * a.prompt, layer.hidden, device="cuda").bfloat16()
    layer.step(x, torch.full((R,), a.prompt, dtype=torch.int32, device="cuda"), layer.buffers(R * a.prompt))
    # one token a request, captured once
    x, one, b = torch.randn(R, layer.hidden, device="cuda").bfloat16(), torch.ones(R, dtype=torch.int32, device="cuda"), layer.buffers(R)
    layer.step(x, one, b, single=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, one, b, single=True)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    graph.replay()
    t0.record()
    for _ in range(a.steps):
        graph.replay()
    t1.record()
    t1.synchronize()
    layer.check()
    us = t0.elapsed_time(t1) * 1e3 / a.steps
    print(f"{R} requests, {int(layer.lengths[0])} tokens each: {us:.1f} us a decoding step of one layer")


if __name__ == "__main__":
    main()
