"""The entry points around a mixture-of-experts block together, as they are
used: the example layer (examples/moe_layer.py) stage by stage against 64 bits,
launched in a row and replayed from a graph, and the gradients of a whole block
against autograd in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import moe_ref
from conftest import ROOT
from gpu_util import DEV, check_y, qtensor_host
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _example():
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("tokens", [1, 13, 300])
def test_layer_stage_by_stage(orc, tokens):
    """Every stage against 64 bits on what the stage before it left."""
    E, k, hidden, width = 6, 2, 256, 128
    layer = _example().MoELayer(hidden=hidden, width=width, experts=E, top_k=k)
    x = (torch.randn(tokens, hidden, generator=torch.Generator().manual_seed(tokens)) * 2).bfloat16()
    b = layer.buffers(tokens)
    y = layer.step(x.to(DEV), b)
    layer.check()
    n, want = b["n"].double().cpu(), moe_ref.norm(x.double(), layer.norm.double().cpu(), None, 1e-6, True)[0]
    assert ((n - want).abs() <= moe_ref.norm_bound(x.double(), layer.norm.double().cpu(), None, 1e-6, True, BF16)[0]).all()
    ids, weights = moe_ref.route(b["logits"].double().cpu(), k, True)
    assert torch.equal(b["ids"].cpu(), ids)
    rel = moe_ref.softmax_over(b["logits"].double().cpu(), ids, True)[1].gather(1, ids.long())
    assert ((b["weights"].double().cpu() - weights).abs() <= weights * rel).all()
    off, row_of, pair_of, fits = moe_ref.sort(ids, E, 128, b["pair_of"].numel())
    assert fits and torch.equal(b["off"].cpu(), off) and torch.equal(b["row_of"].cpu(), row_of) and torch.equal(b["pair_of"].cpu(), pair_of)
    there = pair_of.numpy() >= 0
    expert = ids.flatten().numpy()[pair_of.numpy()[there]]

    def product(pair, w, out, N):
        """The rows of pairs against their experts' dequantized weights."""
        a = sum(orc.dequant(orc.FMT_MXFP4, *qtensor_host(q), q.rows, q.k) for q in pair)
        wv = orc.dequant(orc.FMT_MXFP4, *qtensor_host(w), w.rows, w.k).reshape(E, N, w.k)
        want = np.stack([wv[e] @ r for e, r in zip(expert, a[there])])
        check_y(out.double().cpu().numpy()[there], want, bf16=True)
    token = pair_of.numpy()[there] // k
    o = orc.quantize_act(_bits(b["n"]))
    for q, name in zip(b["x"], ("main", "res")):
        codes, scales = qtensor_host(q)
        assert np.array_equal(codes[there], o[name + "_codes"][token]) and np.array_equal(scales[there], o[name + "_scales"][token])
        assert (codes[~there] == 0).all() and (scales[~there] == 0).all()
    product(b["x"], layer.gate_up, b["gu"], 2 * width)
    assert (b["gu"].cpu()[~there] == 0).all()
    product(b["hq"], layer.down, b["d"], hidden)
    terms = b["weights"].double().cpu()[..., None] * b["d"].double().cpu()[row_of.long()]
    # the combined row is rounded to bf16, then its sum with x once more
    c, e = terms.sum(1), (k + 1) * moe_ref.U * terms.abs().sum(1)
    e = e + moe_ref.half_step(BF16) * (c.abs() + e)
    want = x.double() + c
    assert ((y.double().cpu() - want).abs() <= e + moe_ref.half_step(BF16) * (want.abs() + e)).all()


def test_in_a_row_and_from_a_graph():
    """Kernels of a step may start before the ones in front have finished: the
    same bits with waits between the calls, without, and from a graph."""
    layer = _example().MoELayer(hidden=256, width=128, experts=16, top_k=4)
    x0 = torch.randn(77, 256, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)

    def steps(run, b, rounds=12):
        x = x0.clone()
        for _ in range(rounds):
            x = (run(x, b) * 0.7).contiguous()
        torch.cuda.synchronize()
        return x

    def with_waits(x, b):
        names = ("rfq_norm", "rfq_route", "rfq_moe_sort", "rfq_moe_quantize", "rfq_linear_grouped", "rfq_quantize_act", "rfq_moe_combine")
        kept = {n: getattr(rfq, n) for n in names}

        def waiting(f):
            def call(*a, **kw):
                torch.cuda.synchronize()
                f(*a, **kw)
                torch.cuda.synchronize()
            return call
        try:
            for n, f in kept.items():
                setattr(rfq, n, waiting(f))
            return layer.step(x, b)
        finally:
            for n, f in kept.items():
                setattr(rfq, n, f)
    want = steps(with_waits, layer.buffers(77))
    assert torch.isfinite(want.float()).all()
    for _ in range(3):
        assert torch.equal(steps(layer.step, layer.buffers(77)), want)
    # two graphs with buffers of their own, replayed in turn
    graphs = []
    for _ in range(2):
        b, x = layer.buffers(77), x0.clone()
        layer.step(x, b)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            layer.step(x, b)
        graphs.append((g, x, b))
    for g, x, b in graphs:
        x.copy_(x0)
    for _ in range(12):
        for g, x, b in graphs:
            g.replay()
            x.copy_(b["y"] * 0.7)
    torch.cuda.synchronize()
    for g, x, b in graphs:
        assert torch.equal(x, want)
    layer.check()


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradients_of_a_block(kind, normalize):
    """norm -> router -> experts -> back, in fp32, its gradients put together
    from the entry points', against autograd in 64 bits.  Eight stages, each of
    whose sums of up to 96 terms is off by (CHAIN + 16) u of the terms'
    magnitudes, which is ten times the sum where signs are mixed: 8 x 10 x 144 u
    = 7e-4 of each gradient's norm."""
    g = torch.Generator().manual_seed(7)
    T, D, E, k, align = 45, 96, 6, 2, 8
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x, w, bias = rnd(T, D), 1 + 0.2 * rnd(D), 0.1 * rnd(D)
    router, experts, dout = rnd(D, E) * D ** -0.5, rnd(E, D, D) * D ** -0.5, rnd(T, D)
    rms = kind == "rms"
    K = rfq.RFQ_NORM_RMS if rms else rfq.RFQ_NORM_LAYER
    d = lambda t: t.to(DEV)  # noqa: E731
    new = lambda *s, t=F32: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
    # forward
    n, mean, rstd = new(T, D), new(T), new(T)
    rfq.rfq_norm(d(x), n, weight=d(w), bias=d(bias), kind=K, mean=mean, rstd=rstd)
    logits = n @ d(router)
    ids, weights = new(T, k, t=I32), new(T, k)
    rfq.rfq_route(logits, ids, weights, normalize=normalize)
    rows = rfq.rfq_moe_rows(T, k, E, align)
    off, row_of, pair_of, ws = new(E + 1, t=I32), new(T, k, t=I32), new(rows, t=I32), torch.zeros(64, dtype=I32, device=DEV)
    rfq.rfq_moe_sort(ids, off, row_of, pair_of, ws, align=align)
    xs, ys, out = new(rows, D), torch.zeros(rows, D, device=DEV), new(T, D)
    rfq.rfq_moe_gather(n, row_of, xs, pair_of=pair_of)
    o = off.tolist()
    for e in range(E):
        ys[o[e]:o[e + 1]] = xs[o[e]:o[e + 1]] @ d(experts)[e]
    rfq.rfq_moe_combine(ys, row_of, out, weights=weights)
    # backward
    dys, dweights = new(rows, D), new(T, k)
    rfq.rfq_moe_combine_grad(d(dout), ys, row_of, weights, dys, dweights, pair_of=pair_of)
    dxs, dexperts = torch.zeros(rows, D, device=DEV), new(E, D, D)
    for e in range(E):
        dxs[o[e]:o[e + 1]] = dys[o[e]:o[e + 1]] @ d(experts)[e].t()
        dexperts[e] = xs[o[e]:o[e + 1]].t() @ dys[o[e]:o[e + 1]]
    dn = new(T, D)
    rfq.rfq_moe_combine(dxs, row_of, dn)
    dlogits = torch.empty_like(logits)
    rfq.rfq_route_grad(logits, ids, dweights, dlogits, normalize=normalize)
    drouter = n.t() @ dlogits
    dn += dlogits @ d(router).t()
    dx, dw, db = new(T, D), new(D), new(D)
    rfq.rfq_norm_grad(dn, d(x), rstd, dx, mean=mean, weight=d(w), dweight=dw, dbias=db, workspace=rfq.norm_workspace(D), kind=K)
    assert rfq.rfq_workspace_status(ws) == rfq.RFQ_OK
    # the same block by autograd
    X, W, B, R, Ex = (t.double().requires_grad_() for t in (x, w, bias, router, experts))
    N = moe_ref.norm(X, W, B, 1e-6, rms)[0]
    p = torch.softmax(N @ R, -1).gather(1, ids.cpu().long())
    p = p / p.sum(-1, keepdim=True) if normalize else p
    want = (torch.einsum("td,tkde->tke", N, Ex[ids.cpu().long()]) * p[..., None]).sum(1)
    want.backward(dout.double())
    near = lambda a, c: (a.double().cpu() - c).norm() <= 7e-4 * c.norm()  # noqa: E731
    assert near(out, want.detach())
    for a, c in ((dx, X), (dw, W), (db, B), (drouter, R), (dexperts, Ex)):
        assert near(a, c.grad)


def test_offsets_past_32_bits():
    """Stacked rows and strides whose elements lie beyond 2^31."""
    dim, rows = 4096, 2 ** 20 + 64                     # 8.6 GB in bf16
    y = torch.empty(rows, dim, dtype=BF16, device=DEV)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(4, dim, generator=g).bfloat16().to(DEV)
    row_of = torch.tensor([[0, rows - 1], [2 ** 19, 2 ** 19 + 1], [rows - 2, 5], [2 ** 20, -1]], dtype=I32, device=DEV)
    rfq.rfq_moe_gather(x, row_of, y)
    for t in range(4):
        for r in row_of[t].tolist():
            assert r < 0 or torch.equal(y[r], x[t])
    out = torch.empty_like(x)
    rfq.rfq_moe_combine(y, row_of, out, weights=torch.full((4, 2), 0.5, device=DEV))
    assert torch.equal(out[:3], x[:3]) and torch.equal(out[3], (x[3].float() * 0.5).bfloat16())
    dy, dw = y, torch.empty(4, 2, device=DEV)
    rfq.rfq_moe_combine_grad(x, y, row_of, torch.full((4, 2), 2.0, device=DEV), dy, dw)
    for t in range(4):
        for r in row_of[t].tolist():
            assert r < 0 or torch.equal(dy[r].float(), 2 * x[t].float())
    # three rows of a norm, 2^31 elements apart
    far = y.view(-1).as_strided((3, dim), (2 ** 31 - 2 ** 12, 1))
    far.copy_(x[:3])
    near, y1, y2 = x[:3].contiguous(), torch.empty_like(far.contiguous()), torch.empty(3, dim, dtype=BF16, device=DEV)
    m, r = torch.empty(3, device=DEV), torch.empty(3, device=DEV)
    rfq.rfq_norm(far, y1, mean=m, rstd=r)
    rfq.rfq_norm(near, y2)
    assert torch.equal(y1, y2)
    rfq.rfq_norm_grad(far, far, r, far, mean=m)
    rfq.rfq_norm_grad(near, near, r, y2, mean=m)
    assert torch.equal(far, y2)
    # codes past 2^31: 2^20 rows of 2048 bytes
    q = rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, rows, dim)
    ref = rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, 4, dim)
    rfq.rfq_moe_quantize(x, row_of, q)
    rfq.rfq_quantize_act(x, ref, None, mode=rfq.RFQ_FALLBACK_NONE)
    c, want = q.codes[:rows * dim // 2].view(rows, -1), qtensor_host(ref)[0]
    for t in range(4):
        for r in row_of[t].tolist():
            assert r < 0 or np.array_equal(c[r].cpu().numpy(), want[t])
