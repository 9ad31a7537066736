"""rfq_norm and rfq_norm_grad against float64, within bounds counted from fp32's
roundings (tests/moe_ref.py)."""
import pytest
import torch

import moe_ref
from gpu_util import DEV, guarded_empty, guarded_full
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
KINDS = {"layer": rfq.RFQ_NORM_LAYER, "rms": rfq.RFQ_NORM_RMS}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _x(g, shape, dtype, shift=0.3):
    x = torch.randn(shape, generator=g) * (1 + 15 * (torch.rand(shape[-1], generator=g) < 0.05).float()) + shift
    return x.to(dtype)


def _within(got, want, bound):
    got = got.double().cpu()
    assert got.shape == want.shape
    worst = ((got - want).abs() / bound.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    assert ((got - want).abs() <= bound).all(), f"{worst:.3g} times the bound"


def _check(tokens, heads, row, dim, kind, affine, dtype, wtype, seed=0, shift=0.3, eps=1e-6):
    g, rms = _gen(seed), kind == "rms"
    packed = _x(g, (tokens, row, dim), dtype, shift)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(wtype) if affine else None
    b = (0.3 * torch.randn(dim, generator=g)).to(wtype) if affine == "both" else None
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    f64 = lambda t: None if t is None else t.double()  # noqa: E731
    x = dev(packed)[:, :heads]
    y = guarded_full((tokens, heads, dim), float("nan"), dtype)
    mean, rstd = guarded_full((tokens, heads), float("nan"), F32), guarded_full((tokens, heads), float("nan"), F32)
    rfq.rfq_norm(x, y, weight=dev(w), bias=dev(b), kind=KINDS[kind], eps=eps, mean=mean, rstd=rstd)
    x64 = packed[:, :heads].double()
    want = moe_ref.norm(x64, f64(w), f64(b), eps, rms)
    for a, c, e in zip((y, mean, rstd), want, moe_ref.norm_bound(x64, f64(w), f64(b), eps, rms, dtype)):
        _within(a, c, e)
    # the gradient, from the statistics that the forward pass left
    dyp = torch.randn(tokens, row, dim, generator=g).to(dtype)
    dy = dev(dyp)[:, :heads]
    dx, dw, db = guarded_full((tokens, heads, dim), float("nan"), dtype), guarded_full((dim,), float("nan"), F32), guarded_full((dim,), float("nan"), F32)
    ws = rfq.norm_workspace(dim)
    rfq.rfq_norm_grad(dy, x, rstd, dx, mean=None if rms else mean, weight=dev(w), dweight=dw, dbias=db, workspace=ws, kind=KINDS[kind])
    args = dyp[:, :heads].double(), x64, mean.double().cpu(), rstd.double().cpu(), f64(w), rms
    for a, c, e in zip((dx, dw, db), moe_ref.norm_grad(*args), moe_ref.norm_grad_bound(*args, dtype)):
        _within(a, c, e)
    # again, in place, and without the weight's gradient: the same bits
    dw2 = torch.empty_like(dw)
    again = dyp[:, :heads].contiguous().to(DEV)
    rfq.rfq_norm_grad(again, x, rstd, again, mean=None if rms else mean, weight=dev(w), dweight=dw2, workspace=ws, kind=KINDS[kind])
    assert torch.equal(again, dx) and torch.equal(dw2, dw)
    alone = torch.empty_like(dx)
    rfq.rfq_norm_grad(dy, x, rstd, alone, mean=None if rms else mean, weight=dev(w), kind=KINDS[kind])
    assert torch.equal(alone, dx)
    same = packed[:, :heads].contiguous().to(DEV)
    rfq.rfq_norm(same, same, weight=dev(w), bias=dev(b), kind=KINDS[kind], eps=eps)
    assert torch.equal(same, y)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype,wtype", [(BF16, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("tokens,dim", [(1, 1), (1, 8), (3, 5), (7, 64), (61, 80), (300, 128), (33, 256), (9, 1000), (5, 1023), (13, 2048),
                                        (700, 5120), (500, 8288), (400, 12296), (3, 13824), (2, 16383), (2, 16384)])
def test_rows(kind, dtype, wtype, tokens, dim):
    _check(tokens, 1, 1, dim, kind, "both", dtype, wtype, seed=dim)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,dim", [(5, 2), (40, 3), (9, 10), (33, 17), (70, 31), (300, 65), (50, 131), (29, 257), (31, 258), (17, 511), (9, 513), (700, 620),
                                        (7, 2047), (3, 4095), (3, 4097), (5, 4098), (400, 5121), (2, 8193), (3, 10001), (3, 16382)])
def test_rows_of_no_convenient_length(dtype, tokens, dim):
    """Rows that start inside a 16-byte word, or of bf16 inside a 4-byte one."""
    _check(tokens, 1, 1, dim, "layer" if dim % 2 else "rms", "both", dtype, F32 if dim % 3 else dtype, seed=dim)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [1, 6, 33, 75, 300, 1001, 6000])
@pytest.mark.parametrize("heads,row", [(1, 1), (3, 5)])
def test_odd_strides_in_place(dtype, dim, heads, row):
    """Rows of odd strides, the result in the place of its input: what lies
    between the rows stays as it was."""
    g = _gen(dim)
    T, pad = 11, 3
    base = _x(g, (T, row * dim + pad), dtype).to(DEV)
    x = base[:, :row * dim].unflatten(1, (row, dim))[:, :heads]
    dy0 = torch.randn(T, row * dim + pad, generator=g).to(dtype).to(DEV)
    want, before = torch.empty(T, heads, dim, dtype=dtype, device=DEV), base.clone()
    mean, rstd = torch.empty(T, heads, device=DEV), torch.empty(T, heads, device=DEV)
    rfq.rfq_norm(x.contiguous(), want, mean=mean, rstd=rstd)
    x64 = x.double().cpu()
    bound = moe_ref.norm_bound(x64, None, None, 1e-6, False, dtype)[0]
    _within(want, moe_ref.norm(x64, None, None, 1e-6, False)[0], bound)
    keep = torch.ones(T, row * dim + pad, dtype=torch.bool, device=DEV)
    keep[:, :row * dim].unflatten(1, (row, dim))[:, :heads] = False
    dx = dy0.clone()
    there = dx[:, :row * dim].unflatten(1, (row, dim))[:, :heads]
    rfq.rfq_norm_grad(there, x, rstd, there, mean=mean)
    args = dy0[:, :row * dim].unflatten(1, (row, dim))[:, :heads].double().cpu(), x64, mean.double().cpu(), rstd.double().cpu(), None, False
    _within(there, moe_ref.norm_grad(*args)[0], moe_ref.norm_grad_bound(*args, dtype)[0])
    assert torch.equal(dx[keep], dy0[keep])
    rfq.rfq_norm(x, x)
    _within(x, moe_ref.norm(x64, None, None, 1e-6, False)[0], bound)
    assert torch.equal(base[keep], before[keep])


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,heads,row,dim", [(1, 1, 3, 128), (37, 5, 9, 128), (11, 40, 48, 64), (5, 3, 4, 80), (4, 3, 5, 33), (2000, 4, 6, 24)])
def test_heads_of_a_projection(kind, dtype, tokens, heads, row, dim):
    _check(tokens, heads, row, dim, kind, "weight", dtype, dtype, seed=tokens)


@pytest.mark.parametrize("affine", [None, "weight"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_without_weights(affine, dtype):
    _check(29, 1, 1, 520, "layer", affine, dtype, dtype)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_a_mean_far_from_zero(kind):
    """The variance is that of the differences: a mean 1000 times the spread."""
    _check(17, 1, 1, 768, kind, "both", F32, F32, shift=1000.0)


def test_rows_that_lie_anywhere():
    """Strides of a row that are no multiple of 16 bytes, and rows apart."""
    for dtype in (BF16, F32):
        base = _x(_gen(3), (9, 130), dtype).to(DEV)
        x = base[:, :128]                              # stride 130
        y = torch.zeros(9, 141, dtype=dtype, device=DEV)
        out = y[:, :128]
        rfq.rfq_norm(x, out)
        want = torch.empty(9, 128, dtype=dtype, device=DEV)
        rfq.rfq_norm(x.contiguous(), want)
        # (another split of a row over threads sums in another order)
        _within(out, want.double().cpu(), 2 * moe_ref.norm_bound(x.double().cpu(), None, None, 1e-6, False, dtype)[0])
        assert (y[:, 128:] == 0).all()


def test_constant_and_extreme_rows():
    """A constant row has rstd = eps^-1/2 and y = b; rows with Inf or NaN are NaN
    alone; elements whose squares pass fp32 give rstd 0."""
    x = torch.ones(6, 256)
    x[1] = 0
    x[2, 7] = float("inf")
    x[3, 9] = float("nan")
    x[4] = torch.randn(256, generator=_gen(1)) * 1e30
    x = x.to(DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    b = torch.randn(256, generator=_gen(2)).to(DEV)
    rfq.rfq_norm(x, y, bias=b, eps=1e-4, mean=mean, rstd=rstd)
    for r in (0, 1, 5):
        assert torch.equal(y[r], b) and abs(rstd[r].item() - 100) < 1e-3
    assert y[2].isnan().all() and y[3].isnan().all()
    assert rstd[4].item() == 0 and torch.equal(y[4], b)


def test_no_rows():
    x = torch.empty(0, 64, device=DEV)
    y = torch.empty_like(x)
    rfq.rfq_norm(x, y)
    dw, db = torch.full((64,), 3.0, device=DEV), torch.full((64,), 3.0, device=DEV)
    rfq.rfq_norm_grad(x, x, torch.empty(0, device=DEV), y, mean=torch.empty(0, device=DEV), dweight=dw, dbias=db, workspace=rfq.norm_workspace(64))
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradient_against_differences(kind):
    """<dx, v> against central differences of the float64 forward pass."""
    g, rms = _gen(11), kind == "rms"
    x, v, dy = (torch.randn(6, 96, generator=g) for _ in range(3))
    w, wv = 1 + 0.3 * torch.randn(96, generator=g), torch.randn(96, generator=g)
    xd, dx, dw, db = x.to(DEV), torch.empty(6, 96, device=DEV), torch.empty(96, device=DEV), torch.empty(96, device=DEV)
    mean, rstd = torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    rfq.rfq_norm(xd, torch.empty_like(xd), weight=w.to(DEV), kind=KINDS[kind], mean=mean, rstd=rstd)
    rfq.rfq_norm_grad(dy.to(DEV), xd, rstd, dx, mean=mean, weight=w.to(DEV), dweight=dw, dbias=db, workspace=rfq.norm_workspace(96), kind=KINDS[kind])
    f = lambda a, c, d: (moe_ref.norm(a, c, d, 1e-6, rms)[0] * dy.double()).sum()  # noqa: E731
    x, w, v, wv, zero, h = x.double(), w.double(), v.double(), wv.double(), torch.zeros(96, dtype=torch.float64), 1e-4
    args = dy.double(), x, mean.double().cpu(), rstd.double().cpu(), w, rms
    ex, ew, eb = moe_ref.norm_grad_bound(*args, F32)
    # (h^2 times a third derivative of a few hundred: 1e-5 of sums of some tens; the statistics are off by 1e-5 of themselves at most)
    for got, along, e, num in ((dx, v, ex, f(x + h * v, w, zero) - f(x - h * v, w, zero)), (dw, wv, ew, f(x, w + h * wv, zero) - f(x, w - h * wv, zero)),
                               (db, wv, eb, f(x, w, zero + h * wv) - f(x, w, zero - h * wv))):
        have = (got.double().cpu() * along).sum()
        assert (have - num / (2 * h)).abs() <= (e * along.abs()).sum() + 1e-5 * (got.double().cpu() * along).abs().sum() + 1e-4


def test_other_stream_and_graph():
    """On a stream of the caller's, and replayed from a graph with new inputs."""
    g = _gen(5)
    x = _x(g, (50, 640), BF16).to(DEV)
    dy = torch.randn(50, 640, generator=g).bfloat16().to(DEV)
    w = (1 + 0.1 * torch.randn(640, generator=g)).bfloat16().to(DEV)
    ws = rfq.norm_workspace(640)
    new = lambda: [torch.empty_like(x), torch.empty(50, device=DEV), torch.empty(50, device=DEV), torch.empty_like(x), torch.empty(640, device=DEV)]  # noqa: E731

    def both(y, mean, rstd, dx, dw, stream=None):
        rfq.rfq_norm(x, y, weight=w, mean=mean, rstd=rstd, stream=stream)
        rfq.rfq_norm_grad(dy, x, rstd, dx, mean=mean, weight=w, dweight=dw, workspace=ws, stream=stream)
    want, got, cap = new(), new(), new()
    both(*want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    both(*got, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        both(*cap)
    x.copy_(_x(_gen(6), (50, 640), BF16))
    graph.replay()
    both(*want)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(cap, want))
