"""rfq_route and rfq_route_grad against float64: choices exactly, weights and
gradients within bounds counted from fp32's roundings (tests/moe_ref.py)."""
import pytest
import torch

import moe_ref
from gpu_util import DEV, guarded_full
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")


def _logits(seed, T, E, dtype, masked):
    g = torch.Generator().manual_seed(seed)
    l = (2 * torch.randn(T, E, generator=g)).to(dtype)
    if masked:
        l[torch.rand(T, E, generator=g) < 0.3] = -INF
        l[T // 2] = -INF                               # no expert at all
        l[0, :max(1, E - 1)] = -INF                    # one expert
    return l


def _within(got, want, bound):
    """NaN where the reference has NaN, and near it elsewhere."""
    got = got.double().cpu()
    assert torch.equal(got.isnan(), want.isnan())
    assert ((got - want).abs() <= bound)[~want.isnan()].all()


def _check(l, top_k, normalize, dw=None):
    T, E = l.shape
    dtype = l.dtype
    ids, w = guarded_full((T, top_k), 77, torch.int32), guarded_full((T, top_k), float("nan"), F32)
    rfq.rfq_route(l.to(DEV), ids, w, normalize=normalize)
    want_ids, want_w = moe_ref.route(l.double(), top_k, normalize)
    ids_h = ids.cpu()
    assert torch.equal(ids_h, want_ids)
    p, rel = moe_ref.softmax_over(l.double(), want_ids, normalize)
    at = want_ids.long().clamp_min(0)
    bound = want_w * rel.gather(1, at) + 2.0 ** -149
    _within(w, want_w, bound)
    if dw is None:
        dw = torch.randn(T, top_k, generator=torch.Generator().manual_seed(T))
    dl = guarded_full((T, E), float("nan"), dtype)
    rfq.rfq_route_grad(l.to(DEV), ids, dw.to(DEV), dl, normalize=normalize)
    want, bound = moe_ref.route_grad(l.double(), want_ids, dw.double(), normalize)
    _within(dl, want, bound + moe_ref.half_step(dtype) * (want.abs() + bound))
    # in place of the logits: the same bits
    same = l.to(DEV)
    rfq.rfq_route_grad(same, ids, dw.to(DEV), same, normalize=normalize)
    assert torch.equal(same.nan_to_num(77.0), dl.nan_to_num(77.0))


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 8, 2), (7, 31, 5), (9, 32, 32), (5, 33, 1), (61, 60, 6), (300, 128, 8), (33, 129, 8), (20, 256, 8),
                                   (20, 255, 32)])
def test_route(T, E, k, masked, dtype, normalize):
    _check(_logits(E + k, T, E, dtype, masked), k, normalize)


@pytest.mark.parametrize("normalize", [False, True])
def test_ties_and_extremes(normalize):
    """Equal logits go to the lowest expert; 0 and -0 are equal; logits far apart."""
    l = torch.zeros(6, 100)
    l[1, 50:] = -0.0
    l[2, ::7] = 3.0
    l[3] = -1e30
    l[4, 40] = 300.0
    l[5] = torch.linspace(-3e38, 3e38, 100)            # (its step passes fp32: -inf, and a NaN at the end)
    _check(l, 9, normalize)


@pytest.mark.parametrize("normalize", [False, True])
def test_logits_far_apart(normalize):
    l = torch.tensor([3e38, -3e38, 1e38, 0.0, -1e-38, 87.0, -88.0, 1e-45])
    _check(torch.stack((l, -l, l * 1e-36)), 5, normalize)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("E", [5, 33, 64, 100, 129, 256])
def test_few_values(dtype, E):
    """Rows of few different logits, equal ones in one lane and across lanes: by their experts."""
    g = torch.Generator().manual_seed(E)
    values = torch.tensor([-INF, torch.finfo(dtype).min, -1.0, -0.0, 0.0, torch.finfo(dtype).smallest_normal, 1.0, 1.0078125], dtype=dtype)
    for k in (1, min(7, E), min(32, E)):
        _check(values[torch.randint(0, 8, (70, E), generator=g)], k, True)
        _check(values[torch.randint(3, 5, (3, E), generator=g)], k, False)


def test_nan_among_bf16():
    """NaN of either sign counts as the largest, then +inf."""
    l = torch.randn(4, 64, generator=torch.Generator().manual_seed(1)).to(BF16)
    l[1, 9], l[2, 5], l[3, 60] = float("nan"), INF, INF
    l[3, 7] = torch.tensor([0xFFC0 - 0x10000], dtype=torch.int16).view(BF16)[0]
    l[3, 3] = float("nan")
    ids, w = torch.empty(4, 3, dtype=torch.int32, device=DEV), torch.empty(4, 3, device=DEV)
    for normalize in (False, True):
        rfq.rfq_route(l.to(DEV), ids, w, normalize=normalize)
        assert ids[1, 0].item() == 9 and ids[2, 0].item() == 5 and ids[3].tolist() == [3, 7, 60]
        assert w[1].isnan().all() and w[2].isnan().any() and w[3].isnan().all() and w[0].isfinite().all()


def test_nan_and_inf():
    l = torch.randn(4, 64, generator=torch.Generator().manual_seed(1))
    l[1, 9] = float("nan")
    l[2, 5] = INF
    ids, w = torch.empty(4, 4, dtype=torch.int32, device=DEV), torch.empty(4, 4, device=DEV)
    for normalize in (False, True):
        rfq.rfq_route(l.to(DEV), ids, w, normalize=normalize)
        assert ids[1, 0].item() == 9 and ids[2, 0].item() == 5 and ((ids >= 0) & (ids < 64)).all()
        assert w[1].isnan().all() and w[2].isnan().any() and w[0].isfinite().all() and w[3].isfinite().all()


def test_strided_rows_and_foreign_ids():
    """Rows apart; ids outside the experts and their gradients are not looked at."""
    base = _logits(3, 11, 80, F32, False).to(DEV)
    l = base[:, 3:67]
    ids, w = torch.empty(11, 4, dtype=torch.int32, device=DEV), torch.empty(11, 4, device=DEV)
    with pytest.raises(rfq.RFQError):                 # (starts 12 bytes off)
        rfq.rfq_route(l, ids, w)
    l = base[:, 4:68]
    rfq.rfq_route(l, ids, w)
    ids2, w2 = torch.empty_like(ids), torch.empty_like(w)
    rfq.rfq_route(l.contiguous(), ids2, w2)
    assert torch.equal(ids, ids2) and torch.equal(w, w2)
    dw = torch.randn(11, 4, device=DEV)
    for foreign in (-1, -5, 64, 2 ** 31 - 1):
        ids[:, 1], ids2[:, 1] = foreign, -1
        dw2 = dw.clone()
        dw[:, 1] = float("nan")
        out = torch.zeros(11, 70, device=DEV)
        rfq.rfq_route_grad(l, ids, dw, out[:, :64])
        want, bound = moe_ref.route_grad(l.double().cpu(), ids2.cpu(), torch.where(ids2 >= 0, dw2, 0.0).double().cpu(), True)
        assert ((out[:, :64].double().cpu() - want).abs() <= bound + moe_ref.half_step(F32) * want.abs()).all() and (out[:, 64:] == 0).all()
        dw = dw2


@pytest.mark.parametrize("normalize", [False, True])
def test_gradient_against_differences(normalize):
    g = torch.Generator().manual_seed(4)
    l, dw, v = torch.randn(5, 20, generator=g), torch.randn(5, 3, generator=g), torch.randn(5, 20, generator=g).double()
    ids, w, dl = torch.empty(5, 3, dtype=torch.int32, device=DEV), torch.empty(5, 3, device=DEV), torch.empty(5, 20, device=DEV)
    rfq.rfq_route(l.to(DEV), ids, w, normalize=normalize)
    rfq.rfq_route_grad(l.to(DEV), ids, dw.to(DEV), dl, normalize=normalize)
    at = ids.cpu().long()

    def f(a):
        p = torch.softmax(a, -1).gather(1, at)
        return ((p / p.sum(-1, keepdim=True) if normalize else p) * dw.double()).sum()
    l, h = l.double(), 1e-5
    num = (f(l + h * v) - f(l - h * v)) / (2 * h)
    have = (dl.double().cpu() * v).sum()
    # fp32's own share (below 1e-5 of the terms) and h^2 of third derivatives of order one
    assert (have - num).abs() <= 1e-5 * (dl.double().cpu() * v).abs().sum() + 1e-7


def test_no_tokens_and_graph():
    l = torch.empty(0, 16, device=DEV)
    rfq.rfq_route(l, torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(0, 2, device=DEV))
    l = _logits(1, 40, 128, F32, False).to(DEV)
    ids, w, dl = torch.empty(40, 8, dtype=torch.int32, device=DEV), torch.empty(40, 8, device=DEV), torch.empty_like(l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rfq.rfq_route(l, ids, w)
        rfq.rfq_route_grad(l, ids, w, dl)
    l.copy_(_logits(2, 40, 128, F32, True))
    graph.replay()
    ids2, w2, dl2 = torch.empty_like(ids), torch.empty_like(w), torch.empty_like(dl)
    rfq.rfq_route(l, ids2, w2)
    rfq.rfq_route_grad(l, ids2, w2, dl2)
    assert torch.equal(ids, ids2) and torch.equal(w, w2) and torch.equal(dl, dl2)
