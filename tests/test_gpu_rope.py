"""rfq_rope against the rotation in 64 bits, its gradient against the formula
and against differences."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import DEV, guarded_empty
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
# One rounding of the result (unit roundoff 2^-24 and 2^-8; fp32: three roundings of the products and sum,
# and 2 ulp each of sine and cosine): relative to the pair's length.
TOL = {torch.float32: 8 * 2.0 ** -24, torch.bfloat16: 2.0 ** -8 + 8 * 2.0 ** -24}


def _tables(P, axes, seed):
    rng = np.random.default_rng(seed)
    freq = (10000.0 ** (-np.arange(P) / P)).astype(np.float32)
    return freq, rng.integers(0, axes, P).astype(np.int32)


def _run(x, pos, freq, axis, pairing, inverse, out=None):
    out = x if out is None else out
    rfq.rfq_rope(x, out, torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV), torch.from_numpy(axis).to(DEV),
                 pairing=pairing, inverse=inverse)
    return out


def _check(got, want, x, P, pairing, dtype):
    got, x = got.double().cpu().numpy(), x.double().cpu().numpy()
    a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if pairing else (x[..., :P], x[..., P:2 * P])
    length = np.sqrt(a * a + b * b)
    length = np.repeat(length, 2, -1) if pairing else np.concatenate([length, length], -1)
    err = np.abs(got - want)
    assert (err[..., :2 * P] <= TOL[dtype] * length + 1e-37).all(), (err[..., :2 * P] / np.maximum(length, 1e-30)).max()
    np.testing.assert_array_equal(got[..., 2 * P:], x[..., 2 * P:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("T,H,D,P,axes", [(1, 1, 128, 64, 3), (5, 40, 128, 64, 3), (1031, 3, 128, 64, 1), (700, 8, 64, 16, 2),
                                          (33, 2, 80, 40, 3), (9, 5, 72, 36, 4), (7, 3, 6, 3, 2), (3, 2, 2, 1, 1), (2, 1, 1024, 512, 3)])
@pytest.mark.parametrize("inverse", [False, True])
def test_matches_the_rotation(dtype, pairing, T, H, D, P, axes, inverse):
    rng = np.random.default_rng(T + D)
    freq, axis = _tables(P, axes, T)
    pos = rng.integers(0, 5000, (axes, T)).astype(np.int32)
    x = torch.from_numpy(rng.standard_normal((T, H, D)) * np.where(rng.random(D) < .1, 50, 1)).to(dtype)
    want = ref.rope(x.double().numpy(), pos, freq.astype(np.float64), axis, pairing == 1, inverse)
    out = guarded_empty((T, H, D), dtype)
    _check(_run(x.to(DEV), pos, freq, axis, pairing, inverse, out), want, x, P, pairing, dtype)


@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_odd_offsets_and_in_place(dtype, pairing):
    """Heads of a packed projection, turned in place; strides that no 16-byte
    access fits; a transposed [heads][tokens] layout."""
    rng = np.random.default_rng(3)
    T, H, D, P = 37, 4, 64, 32
    freq, axis = _tables(P, 3, 1)
    pos = rng.integers(0, 300, (3, T)).astype(np.int32)
    for row, head in ((9 * D, D), (H * (D + 3) + 5, D + 3), (D, T * D)):
        base = torch.from_numpy(rng.standard_normal(T * row + H * head + D)).to(dtype)
        dev = base.to(DEV)
        x = base.as_strided((T, H, D), (row, head, 1))
        want = ref.rope(x.double().numpy(), pos, freq.astype(np.float64), axis, pairing == 1, False)
        got = _run(dev.as_strided((T, H, D), (row, head, 1)), pos, freq, axis, pairing, False)
        _check(got, want, x, P, pairing, dtype)
        keep = torch.ones_like(base, dtype=torch.bool)
        keep.as_strided((T, H, D), (row, head, 1)).fill_(False)
        assert torch.equal(dev.cpu()[keep], base[keep])     # nothing else was written


def test_large_positions_keep_fp32_accuracy():
    T, P = 64, 32
    freq, axis = _tables(P, 1, 0)
    pos = np.linspace(0, 2 ** 31 - 1, T).astype(np.int64).astype(np.int32)[None]
    pos[0, 1] = -1234567
    x = torch.randn(T, 2, 64, dtype=torch.float32)
    want = ref.rope(x.double().numpy(), pos, freq.astype(np.float64), axis, False, False)
    _check(_run(x.to(DEV), pos, freq, axis, 0, False), want, x, P, 0, torch.float32)


def test_axis_outside_leaves_the_pair():
    x = torch.randn(3, 2, 8)
    freq, axis = np.ones(4, np.float32), np.array([0, 7, -1, 1], np.int32)
    pos = np.array([[1, 2, 3], [4, 5, 6]], np.int32)
    want = ref.rope(x.double().numpy(), pos, freq.astype(np.float64), axis, True, False)
    _check(_run(x.to(DEV), pos, freq, axis, 1, False), want, x, 4, 1, torch.float32)


@pytest.mark.parametrize("pairing", [0, 1])
def test_gradient_against_differences(pairing):
    """d/dx of sum(w * rope(x)) by central differences in fp32 equals
    rope^-1(w): the map is linear, so steps of 1 have no truncation error."""
    T, H, D, P = 3, 2, 16, 8
    freq, axis = _tables(P, 2, 5)
    pos = np.array([[3, 70, 900], [1, 2, 50]], np.int32)
    w = torch.randn(T, H, D)
    grad = _run(w.to(DEV).clone(), pos, freq, axis, pairing, True).cpu()
    for t, h, d in ((0, 0, 0), (1, 1, 5), (2, 0, 15), (2, 1, 8)):
        x = torch.zeros(T, H, D)
        f = []
        for step in (1.0, -1.0):
            x[t, h, d] = step
            f.append(float((w.double() * _run(x.to(DEV).clone(), pos, freq, axis, pairing, False).cpu().double()).sum()))
        assert abs((f[0] - f[1]) / 2 - float(grad[t, h, d])) <= 16 * 2.0 ** -24 * float(w.abs().max())


def test_zero_tokens_and_refusals():
    z = torch.empty(0, 2, 8, device=DEV)
    freq, axis = torch.ones(4, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    rfq.rfq_rope(z, z, torch.empty(1, 0, dtype=torch.int32, device=DEV), freq, axis)
    x, pos = torch.zeros(1, 2, 8, device=DEV), torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        rfq.rfq_rope(x.half(), x.half(), pos, freq, axis)
    with pytest.raises(ValueError):
        rfq.rfq_rope(x, x, pos[:, :0], freq, axis)
    with pytest.raises(ValueError):
        rfq.rfq_rope(x.transpose(1, 2), x.transpose(1, 2), pos, freq, axis)
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_rope(x, x, pos, torch.ones(5, device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV))
    assert e.value.status == rfq.RFQ_ERR_SHAPE
