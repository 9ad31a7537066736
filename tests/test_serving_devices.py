"""Host side of the serving calls on several devices of one process: what a
kernel has to be allowed, and what a launch is sized by, belongs to a device."""
import ctypes

import numpy as np
import pytest

from fake_cuda import FakeCuda
from paper_2608_26581_gb300 import rfq


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeCuda(tmp_path_factory.mktemp("fake"))


def _attention(fake, fmt, D, heads, tokens, requests, q_start=None, width=8):
    kv = rfq._KV(fmt, 2, D, 16, 8, 256, 256, 256, 256)
    return fake.lib.rfq_kv_attention(256, heads * D, D, tokens, heads, q_start, 256, requests, ctypes.byref(kv), 256, width, 0.125, 0,
                                     256, 256, 256, None)


def _matvec(fake, fmt, rows, n, k):
    return fake.lib.rfq_matvec(256, k, rows, ctypes.byref(rfq._QT(fmt, 1, n, k, 256, 256)), 256, 0, None)


@pytest.mark.parametrize("fmt", [rfq.RFQ_FMT_MXFP4, rfq.RFQ_FMT_HIF4])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_on_each_device(fake, fmt, D):
    for device in (0, 1, 0, 2):
        fake.device(device)
        sms = 76 if device == 1 else 152
        for heads, tokens, requests, start in ((8, 3, 3, None), (32, 3, 3, None), (80, 3, 3, None), (8, 300, 3, 256)):
            before = len(fake.launches())
            assert _attention(fake, fmt, D, heads, tokens, requests, start) == rfq.RFQ_OK
            assert all(l[0] == sms for l in fake.launches()[before:])


@pytest.mark.parametrize("fmt", [rfq.RFQ_FMT_MXFP4, rfq.RFQ_FMT_HIF4])
@pytest.mark.parametrize("rows", [1, 2, 4, 8, 13, 32])
def test_matvec_on_each_device(fake, fmt, rows):
    for device in (0, 1, 0, 2):
        fake.device(device)
        sms = 76 if device == 1 else 152
        for n, k in ((4096, 12288), (8192, 4096), (100, 512)):
            before = len(fake.launches())
            assert _matvec(fake, fmt, rows, n, k) == rfq.RFQ_OK
            (x, y, _, _, cluster, _), = fake.launches()[before:]
            # one wave of this device's clusters, where that many hold the tiles
            assert x == cluster and x * y <= sms


def test_the_work_that_is_taken(fake):
    """What the kernels can count is taken: prompts by tiles of 128 rows, tokens
    by tiles of 8; more is refused."""
    fake.device(0)
    kv = rfq._KV(rfq.RFQ_FMT_MXFP4, 8, 128, 64, 2 ** 20, 256, 256, 256, 256)

    def call(tokens, requests, q_start, keys, heads=64):
        return fake.lib.rfq_kv_attention(256, heads * 128, 128, tokens, heads, q_start, 256, requests, ctypes.byref(kv), 256, keys // 64,
                                         0.125, 0, 256, 256, 256, None)
    assert call(131072, 1, 256, 131072) == rfq.RFQ_OK                 # a prompt of as many tokens
    assert call(262144, 64, 256, 131072) == rfq.RFQ_OK                # many of 4096
    assert call(1024, 1024, None, 2 ** 20) == rfq.RFQ_OK              # one token each of long requests
    assert call(1024, 1024, None, 2 ** 20, heads=8 * 128) == rfq.RFQ_OK
    assert call(131072, 1, 256, 2 ** 28) == rfq.RFQ_ERR_SHAPE
    assert call(2 ** 15, 2 ** 15, None, 2 ** 20) == rfq.RFQ_ERR_SHAPE
    assert call(2 ** 25, 1, 256, 64) == rfq.RFQ_ERR_SHAPE             # rows past 32 bits


@pytest.mark.parametrize("tokens,heads", [(1, 1), (7, 40), (32760, 40), (2000, 2 ** 22 + 1), (5, 2 ** 31 - 1)])
def test_rope_blocks(fake, tokens, heads):
    """A block's rows are four tokens of at most 65536 heads: their quotient by
    the heads, (r + 1/2) / heads in fp32, then rounds down to r / heads."""
    fake.device(0)
    before = len(fake.launches())
    assert fake.lib.rfq_rope(256, heads * 2, 2, 256, heads * 2, 2, 1, tokens, heads, 2, 256, 1, 256, 256, 1, 0, 0, None) == rfq.RFQ_OK
    (x, y, _, _, _, _), = fake.launches()[before:]
    each = -(-heads // y)
    assert x * 4 >= tokens and y <= 65535 and each <= 65536


def test_the_quotient_of_a_block_s_rows():
    f = np.float32
    for heads in (1, 2, 3, 5, 7, 40, 48, 1000, 4097, 65521, 65535, 65536):
        r = np.arange(4 * heads)
        assert (((r.astype(f) + f(0.5)) * (f(1) / f(heads))).astype(np.int64) == r // heads).all()
