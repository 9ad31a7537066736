"""One mixture-of-experts feed-forward layer with 4-bit experts.

A step of tokens runs

    RMS norm -> router -> pairs sorted by expert -> tokens quantized into their
    experts' rows -> gate/up product -> gated activation -> down product ->
    rows weighted and brought back -> added to the input

with the experts' weights in MXFP4 and their activations in MXFP4 with the RFQ
residual.  The sizes of a step are fixed by its tensors (the experts' groups lie
in as many rows as they can ever take), so it can be captured in a CUDA graph
and replayed whatever the router chooses.

    python examples/moe_layer.py [--tokens 64] [--steps 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_26581_gb300 import rfq  # noqa: E402


class MoELayer:
    """Weights of the layer, random.  The defaults are the feed-forward layer of
    Qwen3-VL-30B-A3B (hidden 2048, 128 experts of width 768, 8 for a token)."""

    def __init__(self, hidden=2048, width=768, experts=128, top_k=8, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.hidden, self.width, self.experts, self.top_k = hidden, width, experts, top_k
        self.norm = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).bfloat16()
        self.router = (torch.randn(hidden, experts, generator=g, device="cuda") * hidden ** -0.5).bfloat16()
        self.gate_up = self._experts(hidden, 2 * width, g)
        self.down = self._experts(width, hidden, g)
        self.ws = torch.zeros(64, dtype=torch.int32, device="cuda")

    def _experts(self, k, n, g):
        """Every expert's [k, n] weight, quantized and stacked."""
        q = rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, self.experts * n, k)
        rfq.rfq_quantize_weight((torch.randn(k, self.experts * n, generator=g, device="cuda") * k ** -0.5).bfloat16(), q)
        return q

    def buffers(self, tokens):
        """The tensors of a step of `tokens` tokens, kept for as long as such steps are run."""
        bf16, i32 = dict(dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.int32, device="cuda")
        rows = rfq.rfq_moe_rows(tokens, self.top_k, self.experts, 128)
        new = lambda k: [rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, rows, k) for _ in range(2)]  # noqa: E731
        # (the grouped product leaves the rows behind the last group alone: zeros, or what a step with more rows left, which no pair reads)
        return {"n": torch.empty(tokens, self.hidden, **bf16), "logits": torch.empty(tokens, self.experts, **bf16),
                "ids": torch.empty(tokens, self.top_k, **i32), "weights": torch.empty(tokens, self.top_k, device="cuda"),
                "off": torch.empty(self.experts + 1, **i32), "row_of": torch.empty(tokens, self.top_k, **i32),
                "pair_of": torch.empty(rows, **i32), "x": new(self.hidden), "gu": torch.zeros(rows, 2 * self.width, **bf16),
                "h": torch.empty(rows, self.width, **bf16), "hq": new(self.width), "d": torch.zeros(rows, self.hidden, **bf16),
                "y": torch.empty(tokens, self.hidden, **bf16)}

    def step(self, x, b):
        """x bf16 [tokens, hidden]; returns the layer's output, a tensor of b."""
        rfq.rfq_norm(x, b["n"], weight=self.norm, kind=rfq.RFQ_NORM_RMS)
        torch.mm(b["n"], self.router, out=b["logits"])
        rfq.rfq_route(b["logits"], b["ids"], b["weights"])
        rfq.rfq_moe_sort(b["ids"], b["off"], b["row_of"], b["pair_of"], self.ws)
        rfq.rfq_moe_quantize(b["n"], b["row_of"], *b["x"], pair_of=b["pair_of"])
        rfq.rfq_linear_grouped(*b["x"], None, 256, b["off"], self.gate_up, 2 * self.width, b["gu"], rfq.RFQ_OUT_BF16, self.ws)
        gate, up = b["gu"][:, :self.width], b["gu"][:, self.width:]
        torch.mul(torch.nn.functional.silu(gate), up, out=b["h"])
        rfq.rfq_quantize_act(b["h"], *b["hq"])
        rfq.rfq_linear_grouped(*b["hq"], None, 256, b["off"], self.down, self.hidden, b["d"], rfq.RFQ_OUT_BF16, self.ws)
        rfq.rfq_moe_combine(b["d"], b["row_of"], b["y"], weights=b["weights"])
        return b["y"].add_(x)

    def check(self):
        """Raises if a step recorded a device status."""
        s = rfq.rfq_workspace_status(self.ws)
        if s != rfq.RFQ_OK:
            raise rfq.RFQError(s, "MoELayer")


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args()
    layer = MoELayer()
    x, b = torch.randn(a.tokens, layer.hidden, device="cuda").bfloat16(), layer.buffers(a.tokens)
    layer.step(x, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, b)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    graph.replay()
    t0.record()
    for _ in range(a.steps):
        graph.replay()
    t1.record()
    t1.synchronize()
    layer.check()
    print(f"{a.tokens} tokens: {t0.elapsed_time(t1) * 1e3 / a.steps:.1f} us a step of one layer")


if __name__ == "__main__":
    main()
