"""rfq_kv_attention against softmax attention in 64 bits over the values that
the cache holds."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import DEV, guarded_empty, guarded_full
from paper_2608_26581_gb300 import rfq
from paper_2608_26581_gb300.synth import bf16_bits_to_f32, f32_to_bf16_bits
from test_gpu_kv_cache import bits_to_dev, new_cache

pytestmark = pytest.mark.gpu


def check(o, lse, want_o, want_lse, vmax):
    """bf16 output: its rounding (2^-8 of the value) and the f16 weights: each
    is off by at most 2^-11 of itself, so the sum by 2^-11 max |v|, plus fp32
    sums (2^-16 covers them).  lse: fp32 sums of fp32 exponentials of fp32
    scores up to some tens: 2^-17 (1 + |lse|)."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    err = np.abs(o - want_o)
    bound = 2.0 ** -8 * np.abs(want_o) + (2.0 ** -11 + 2.0 ** -16) * vmax + 1e-30
    assert (err <= bound).all(), f"worst {np.max(err / bound):.3f} of the bound"
    dead = np.isneginf(want_lse)
    np.testing.assert_array_equal(np.isneginf(lse), dead)
    assert (o[dead] == 0).all()
    e = np.abs(lse[~dead] - want_lse[~dead])
    assert (e <= 2.0 ** -17 * (1 + np.abs(want_lse[~dead]))).all(), e.max()


class Case:
    """Requests of given lengths in a cache whose other slots hold NaN scales
    (MXFP4 byte 255) or huge ones."""

    def __init__(self, fmt, D, H, G, page, lens, new=None, seed=0, vspread=0, poison=True):
        rng = np.random.default_rng(seed)
        self.fmt, self.D, self.H, self.G, self.page, self.lens = fmt, D, H, G, page, list(lens)
        R = len(lens)
        have = [-(-n // page) for n in lens]
        pages = sum(have) + 2
        ids = rng.permutation(pages).astype(np.int32)
        width = max(1, max(have) if have else 1)
        table = np.full((max(R, 1), width), 2 ** 30, np.int32)      # entries past a request's pages are not pages
        self.cache = new_cache(fmt, H, D, page, pages, fill=0xFF if poison else 0x5A)
        at, slots = 0, []
        for r in range(R):
            table[r, :have[r]] = ids[at:at + have[r]]
            at += have[r]
            slots += [int(table[r, j // page]) * page + j % page for j in range(lens[r])]
        T = len(slots)
        kb = rng.standard_normal((T, H, D)) * np.where(rng.random((H, D)) < 0.05, 12, 1)
        vb = rng.standard_normal((T, H, D)) * np.where(rng.random((H, D)) < 0.05, 40, 1)
        if vspread:
            vb *= 2.0 ** rng.integers(-vspread, vspread + 1, (T, H, 1))
        kb, vb = f32_to_bf16_bits(kb.astype(np.float32)), f32_to_bf16_bits(vb.astype(np.float32))
        self.keys, self.values = [], []
        if T:
            s = torch.tensor(slots, device=DEV)
            rfq.rfq_kv_append(bits_to_dev(kb), bits_to_dev(vb), s, self.cache)
            k, v = torch.empty(T, H, D, device=DEV), torch.empty(T, H, D, device=DEV)
            rfq.rfq_kv_read(self.cache, s, k, v)
            k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
        at = 0
        for n in lens:
            self.keys.append(k[at:at + n] if n else np.zeros((0, H, D)))
            self.values.append(v[at:at + n] if n else np.zeros((0, H, D)))
            at += n
        self.table = torch.from_numpy(table[:R]).to(DEV)
        self.new = new or [1] * R
        self.start = np.concatenate([[0], np.cumsum(self.new)])
        T = int(self.start[-1])
        self.qb = f32_to_bf16_bits(rng.standard_normal((T, H * G, D)).astype(np.float32))
        self.vmax = max([np.abs(v).max() for v in self.values if v.size] or [0.0])

    def run(self, window=0, scale=None, ws=None, qbits=None, decode=None):
        qb = self.qb if qbits is None else qbits
        T, Hq, D = qb.shape
        packed = torch.zeros(T, Hq + 2 * self.H, D, dtype=torch.bfloat16, device=DEV)
        packed[:, :Hq] = bits_to_dev(qb)
        out, lse = guarded_full((T, Hq, D), 7.0, torch.bfloat16), guarded_full((T, Hq), 7.0, torch.float32)
        ws = rfq.kv_attention_workspace(Hq, D) if ws is None else ws
        decode = all(n == 1 for n in self.new) if decode is None else decode
        start = None if decode else torch.tensor(self.start, dtype=torch.int32, device=DEV)
        rfq.rfq_kv_attention(packed[:, :Hq], self.cache, self.table, torch.tensor(self.lens, dtype=torch.int32, device=DEV), out, ws,
                             lse=lse, q_start=start, scale=scale, window=window)
        assert rfq.rfq_workspace_status(ws) == rfq.RFQ_OK
        return out, lse

    def check(self, window=0, scale=None, **kw):
        o, lse = self.run(window, scale, **kw)
        q = bf16_bits_to_f32(self.qb if kw.get("qbits") is None else kw["qbits"]).astype(np.float64)
        want = ref.attention(q, self.keys, self.values, self.start, self.lens, self.D ** -0.5 if scale is None else scale, window)
        check(o, lse, *want, self.vmax)


FMTS = pytest.mark.parametrize("fmt", [ref.FMT_MXFP4, ref.FMT_HIF4])


@FMTS
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 8, 16, 40])
def test_decode_ragged(fmt, D, G):
    Case(fmt, D, 2, G, 16, [1, 0, 15, 16, 17, 127, 128, 129, 300, 700], seed=G).check()


@FMTS
@pytest.mark.parametrize("page", [16, 32, 48, 64, 256])
def test_pages(fmt, page):
    Case(fmt, 128, 2, 4, page, [page - 1, page, page + 1, 3 * page + 5, 1], seed=page).check()


@FMTS
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,new", [(1, [5, 1, 40, 0, 9]), (4, [3, 2, 1, 1, 2]), (4, [33, 1, 64, 7, 100]), (5, [2, 3, 2, 3, 2])])
def test_chunks(fmt, D, G, new):
    """Several new tokens a request: causal among themselves; a request without
    any; rows of a tile that straddle tokens."""
    Case(fmt, D, 2, G, 16, [5, 130, 300, 20, 257], new=new, seed=len(new) + G).check(decode=False)


@FMTS
@pytest.mark.parametrize("window", [1, 7, 16, 100, 1000])
def test_windows(fmt, window):
    Case(fmt, 64, 2, 4, 32, [3, 100, 0, 517], seed=window).check(window=window)
    Case(fmt, 128, 1, 4, 16, [30, 257], new=[20, 40], seed=window).check(window=window)


@FMTS
def test_rows_before_the_first_key(fmt):
    """More new tokens than keys: the first rows see nothing."""
    Case(fmt, 64, 2, 2, 16, [3, 0, 1], new=[5, 4, 1], seed=1).check()


@FMTS
def test_long_request_is_split_over_ctas(fmt):
    Case(fmt, 128, 1, 4, 64, [20000, 3], seed=2).check()
    Case(fmt, 64, 8, 1, 16, [4099], seed=3).check()


def test_many_requests():
    rng = np.random.default_rng(0)
    Case(ref.FMT_MXFP4, 64, 1, 2, 16, rng.integers(0, 40, 700).tolist(), seed=4).check()


@FMTS
def test_value_scales_span_many_octaves(fmt):
    """V of one request spans 2^20 between tokens: exact in f16 relative to
    the running power of two; the bound is relative to the largest."""
    Case(fmt, 128, 2, 4, 16, [300, 40], seed=5, vspread=10).check()


@FMTS
def test_extreme_queries(fmt):
    """A hot softmax, tiny and zero queries: the scores come from exact codes
    and q scaled by a power of two."""
    c = Case(fmt, 128, 2, 4, 16, [200, 33], seed=6)
    q = bf16_bits_to_f32(c.qb) * (2.0 ** np.linspace(-100, 3, c.qb.shape[1]))[None, :, None]
    q[1, 3] = 0
    c.check(qbits=f32_to_bf16_bits(q.astype(np.float32)))


def test_scale_zero_and_negative():
    c = Case(ref.FMT_MXFP4, 64, 1, 4, 16, [77], seed=7)
    c.check(scale=0.0)
    c.check(scale=-0.3)


def test_same_bits_twice_and_workspace_reuse():
    c, d = Case(ref.FMT_MXFP4, 128, 2, 4, 16, [5000, 1, 900], seed=8), Case(ref.FMT_HIF4, 128, 2, 4, 16, [3000], seed=9)
    ws = rfq.kv_attention_workspace(8, 128)
    a = c.run(ws=ws)
    d.check(ws=ws)
    for _ in range(3):
        b = c.run(ws=ws)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_bad_device_sizes_set_the_status():
    c = Case(ref.FMT_MXFP4, 64, 1, 2, 16, [20, 30], seed=10, poison=False)
    q = bits_to_dev(c.qb)
    out = guarded_empty(q.shape, torch.bfloat16)

    def status(table, lens, start=None):
        ws = rfq.kv_attention_workspace(2, 64)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        rfq.rfq_kv_attention(q, c.cache, table, i32(lens), out, ws, q_start=None if start is None else i32(start))
        return rfq.rfq_workspace_status(ws)
    assert status(c.table, [20, 30]) == rfq.RFQ_OK
    assert status(c.table, [20, 33]) == rfq.RFQ_ERR_SHAPE               # past the table's two pages
    assert status(c.table, [-1, 30]) == rfq.RFQ_ERR_SHAPE
    assert status(torch.full_like(c.table, 2 ** 30), [20, 30]) == rfq.RFQ_ERR_SHAPE
    assert status(torch.full_like(c.table, -1), [20, 30]) == rfq.RFQ_ERR_SHAPE
    assert status(c.table, [20, 30], [0, 3, 2]) == rfq.RFQ_ERR_SHAPE
    assert status(c.table, [20, 30], [0, 1, 5]) == rfq.RFQ_ERR_SHAPE


def test_another_stream():
    c = Case(ref.FMT_MXFP4, 64, 2, 2, 16, [200, 30], seed=11)
    q, want = bits_to_dev(c.qb), c.run()
    out, ws = torch.empty_like(q), rfq.kv_attention_workspace(4, 64)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    rfq.rfq_kv_attention(q, c.cache, c.table, torch.tensor(c.lens, dtype=torch.int32, device=DEV), out, ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want[0])


def test_refusals():
    c = Case(ref.FMT_MXFP4, 64, 2, 2, 16, [20], seed=12)
    q, ws = bits_to_dev(c.qb), rfq.kv_attention_workspace(4, 64)
    lens, out = torch.tensor(c.lens, dtype=torch.int32, device=DEV), torch.empty_like(bits_to_dev(c.qb))
    for args in ((q.float(), c.cache, c.table, lens, out, ws), (q, c.cache, c.table, lens.long(), out, ws),
                 (q, c.cache, c.table, lens, out.float(), ws), (q, c.cache, c.table, lens, out, ws[:64])):
        with pytest.raises(ValueError):
            rfq.rfq_kv_attention(*args)
    q3 = torch.zeros(1, 3, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_kv_attention(q3, c.cache, c.table, lens, torch.empty_like(q3), ws)
    assert e.value.status == rfq.RFQ_ERR_SHAPE
    with pytest.raises(rfq.RFQError) as e:
        rfq.rfq_kv_attention(q, c.cache, c.table, lens, out, ws, window=-1)
    assert e.value.status == rfq.RFQ_ERR_SHAPE
