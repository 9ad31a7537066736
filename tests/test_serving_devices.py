"""Host side of the serving calls on several devices of one process: what a
kernel has to be allowed, and what a launch is sized by, belongs to a device."""
import ctypes

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
