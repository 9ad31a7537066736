"""What the header says of the entry points around a mixture-of-experts block,
in calls that lie at the edge of it."""
import importlib.util
import os

import pytest
import torch

import moe_ref
from conftest import ROOT
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


def _rows_and_back(x, dy, w, rms, rstd_mean, dx, dw, db, ws):
    mean, rstd = rstd_mean
    kind = rfq.RFQ_NORM_RMS if rms else rfq.RFQ_NORM_LAYER
    rfq.rfq_norm(x, torch.empty(x.shape, dtype=x.dtype, device=DEV), weight=w, kind=kind, mean=mean, rstd=rstd)
    rfq.rfq_norm_grad(dy, x, rstd, dx, mean=mean, weight=w, dweight=dw, dbias=db, workspace=ws, kind=kind)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,dim,bf16_groups,f32_groups", [(60000, 16, 256, 64), (40001, 128, 32, 16), (9120, 257, 1, 1), (9001, 300, 1, 8), (9120, 511, 1, 1),
                                                              (32760, 512, 8, 8), (12160, 1024, 1, 1), (8001, 1023, 1, 1), (912, 8288, 1, 1), (608, 8193, 1, 1),
                                                              (608, 16384, 1, 1)])
def test_weight_gradients_of_many_rows(rows, dim, bf16_groups, f32_groups, dtype):
    """dweight and dbias over as many rows as the blocks go through in several
    turns, within a bound counted from their chains of additions; nothing is
    written behind a workspace that such a call can fill to its end.

    A block takes `groups` rows at once, and four turns or as many as the rows of
    an SM need: a thread adds the rows of its turns, then the block its groups'
    sums; the second kernel adds a 32nd of at most ten blocks an SM, then 32 sums."""
    g, sms = torch.Generator().manual_seed(dim), torch.cuda.get_device_properties(0).multi_processor_count
    x, dy = (torch.randn(rows, dim, generator=g) + 0.3).to(dtype), torch.randn(rows, dim, generator=g).to(dtype)
    w = 1 + 0.3 * torch.randn(dim, generator=g)
    groups = bf16_groups if dtype is BF16 else f32_groups
    chain = max(4, -(-rows // (groups * sms))) + groups + -(-10 * sms // 32) + 32
    size = rfq.rfq_norm_grad_workspace_bytes(dim)
    for rms in (False, True):
        stats, dw, db = (torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)), guarded_full((dim,), float("nan"), F32), guarded_full((dim,), float("nan"), F32)
        dx = guarded_full((rows, dim), float("nan"), dtype)
        _rows_and_back(x.to(DEV), dy.to(DEV), w.to(DEV), rms, stats, dx, dw, db, guarded_full((size // 4,), float("nan"), F32))
        args = dy.double(), x.double(), *(s.double().cpu() for s in stats), w.double(), rms
        ex, want = moe_ref.norm_grad_bound(*args, dtype)[0], moe_ref.norm_grad(*args)
        h = (args[1] - (0 if rms else args[2][:, None])) * args[3][:, None]
        # (a term's own roundings: the difference, the product with rstd, and room for products of errors)
        bounds = ex, (chain + 4) * moe_ref.U * (args[0] * h).abs().sum(0), (chain + 1) * moe_ref.U * args[0].abs().sum(0)
        for got, c, e in zip((dx, dw, db), want, bounds):
            assert ((got.double().cpu() - c).abs() <= e).all(), ((got.double().cpu() - c).abs() / e.clamp_min(1e-300)).max()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [128, 33, 600])
def test_strides_in_any_order(dim, dtype):
    """Heads that lie before tokens, and rows that are read several times
    (expanded: strides of 0), give the bits of the same rows lying in order."""
    g = torch.Generator().manual_seed(dim)
    T, H = 37, 5
    heads_first = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    new = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    x, dy = torch.randn(T, H, dim, generator=g).to(dtype).to(DEV), torch.randn(T, H, dim, generator=g).to(dtype).to(DEV)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(DEV)
    ws = rfq.norm_workspace(dim)
    assert heads_first(x).stride() == (dim, T * dim, 1)

    def run(x, dy, place):
        stats, dw, db = (new(T * H), new(T * H)), new(dim), new(dim)
        y, dx = place(torch.full((T, H, dim), float("nan"), dtype=dtype, device=DEV)), place(torch.full((T, H, dim), float("nan"), dtype=dtype, device=DEV))
        rfq.rfq_norm(x, y, weight=w, mean=stats[0], rstd=stats[1])
        rfq.rfq_norm_grad(dy, x, stats[1], dx, mean=stats[0], weight=w, dweight=dw, dbias=db, workspace=ws)
        return y, *stats, dx, dw, db
    for a, b in ((x, dy), (x[:1].expand(T, H, dim), dy), (x[:, :1].expand(T, H, dim), dy), (x, dy[:1, :1].expand(T, H, dim))):
        want = run(a.contiguous(), b.contiguous(), lambda t: t)
        for got in (run(a, b, lambda t: t), run(a, b, heads_first), run(heads_first(a), heads_first(b), heads_first)):
            assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_steps_of_other_routings_in_one_set_of_buffers():
    """What a step with more rows left behind the last group of the next one's
    is not seen by it."""
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    layer = m.MoELayer(hidden=256, width=128, experts=16, top_k=2)
    g = torch.Generator().manual_seed(4)
    spread, alike = torch.randn(60, 256, generator=g).bfloat16().to(DEV), torch.randn(1, 256, generator=g).bfloat16().to(DEV).expand(60, 256).contiguous()
    fresh, used = layer.buffers(60), layer.buffers(60)
    want = layer.step(alike, fresh).clone()
    layer.step(spread, used)
    many = used["off"][-1].item()
    got = layer.step(alike, used)
    layer.check()
    assert used["off"][-1].item() == 256 < many and (used["gu"][256:many] != 0).any() and torch.equal(got, want)


@pytest.mark.parametrize("dim", [64, 1023])
def test_rows_whose_sum_passes_fp32(dim):
    """Finite elements whose sum is none in fp32: NaN in a layer norm, rstd = 0 in
    an RMS norm, and the rows beside them as ever."""
    x = torch.randn(3, dim, generator=torch.Generator().manual_seed(1))
    x[1] = 3e38
    for dtype in (BF16, F32):
        xs, y, rstd = x.to(dtype).to(DEV), torch.empty(3, dim, dtype=dtype, device=DEV), torch.empty(3, device=DEV)
        assert xs.isfinite().all()
        rfq.rfq_norm(xs, y, rstd=rstd)
        assert y[1].isnan().all() and y[[0, 2]].isfinite().all()
        rfq.rfq_norm(xs, y, kind=rfq.RFQ_NORM_RMS, rstd=rstd)
        assert rstd[1].item() == 0 and (y[1] == 0).all() and y[[0, 2]].isfinite().all()
