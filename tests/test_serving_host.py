"""Host-side checks of the serving entry points: every refusal comes before
any device work (the pointers below are not device memory)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2608_26581_gb300 import _build, rfq
    _build.build()
    return rfq.load_library()


def test_cache_bytes(lib):
    from paper_2608_26581_gb300 import rfq
    assert rfq.rfq_kv_cache_bytes(rfq.RFQ_FMT_MXFP4, 8, 128, 16, 10) == (8 * 160 * 64, 8 * 160 * 4)
    assert rfq.rfq_kv_cache_bytes(rfq.RFQ_FMT_HIF4, 8, 128, 16, 10) == (8 * 160 * 64, 8 * 160 * 8)
    assert rfq.rfq_kv_cache_bytes(rfq.RFQ_FMT_HIF4, 1, 64, 4096, 2 ** 20) == (2 ** 32 * 32, 2 ** 32 * 4)
    for args, status in (((2, 8, 128, 16, 10), rfq.RFQ_ERR_INVALID_ARG), ((0, 0, 128, 16, 1), rfq.RFQ_ERR_SHAPE),
                         ((0, 1, 128, 24, 1), rfq.RFQ_ERR_SHAPE), ((0, 1, 128, 8192, 1), rfq.RFQ_ERR_SHAPE),
                         ((0, 1, 96, 16, 1), rfq.RFQ_ERR_UNSUPPORTED), ((0, 1, 64, 16, -1), rfq.RFQ_ERR_SHAPE)):
        with pytest.raises(rfq.RFQError) as e:
            rfq.rfq_kv_cache_bytes(*args)
        assert e.value.status == status


def test_slot_map_checks(lib):
    from paper_2608_26581_gb300 import rfq
    good = [16, 16, 2, 16, 16, 4, 16, 8, 16, 16, 16, 16, 16, 16, 5, 16, None]

    def call(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return lib.rfq_slot_map(*a)
    assert call(_2=-1) == rfq.RFQ_ERR_SHAPE and call(_2=8193) == rfq.RFQ_ERR_SHAPE
    assert call(_3=0) == rfq.RFQ_ERR_SHAPE and call(_5=0) == rfq.RFQ_ERR_SHAPE and call(_14=-1) == rfq.RFQ_ERR_SHAPE
    for i in (0, 1, 4, 6, 8, 9, 10, 11, 12, 13, 15):
        assert call(**{f"_{i}": None}) == rfq.RFQ_ERR_INVALID_ARG
    assert call(_0=18) == rfq.RFQ_ERR_ALIGNMENT and call(_12=20) == rfq.RFQ_ERR_ALIGNMENT and call(_15=8) == rfq.RFQ_ERR_ALIGNMENT


def test_rope_checks(lib):
    from paper_2608_26581_gb300 import rfq
    good = [16, 256, 64, 16, 256, 64, 1, 3, 4, 64, 16, 3, 16, 16, 32, 0, 0, None]

    def call(i, v):
        a = list(good)
        a[i] = v
        return lib.rfq_rope(*a)
    for i in (0, 3, 10, 12, 13):
        assert call(i, None) == rfq.RFQ_ERR_INVALID_ARG
    assert call(6, 2) == rfq.RFQ_ERR_INVALID_ARG and call(15, 2) == rfq.RFQ_ERR_INVALID_ARG
    for i, v in ((7, -1), (8, 0), (9, 0), (9, 1025), (11, 0), (14, 0), (14, 33), (1, -1)):
        assert call(i, v) == rfq.RFQ_ERR_SHAPE
    assert call(0, 8) == rfq.RFQ_ERR_ALIGNMENT and call(13, 6) == rfq.RFQ_ERR_ALIGNMENT


def test_cache_call_checks(lib):
    from paper_2608_26581_gb300 import rfq
    kv = rfq._KV(0, 2, 64, 16, 3, 16, 16, 16, 16)
    ref = ctypes.byref
    assert lib.rfq_kv_append(16, 128, 64, 16, 128, 64, 3, 16, None, None) == rfq.RFQ_ERR_INVALID_ARG
    assert lib.rfq_kv_append(None, 128, 64, 16, 128, 64, 3, 16, ref(kv), None) == rfq.RFQ_ERR_INVALID_ARG
    assert lib.rfq_kv_append(16, 128, 64, 16, 128, 64, -1, 16, ref(kv), None) == rfq.RFQ_ERR_SHAPE
    assert lib.rfq_kv_append(16, 132, 64, 16, 128, 64, 3, 16, ref(kv), None) == rfq.RFQ_ERR_ALIGNMENT
    assert lib.rfq_kv_append(24, 128, 64, 16, 128, 64, 3, 16, ref(kv), None) == rfq.RFQ_ERR_ALIGNMENT
    assert lib.rfq_kv_read(ref(kv), 16, 3, 16, 16, 2, None) == rfq.RFQ_ERR_INVALID_ARG
    assert lib.rfq_kv_read(ref(kv), 20, 3, 16, 16, 1, None) == rfq.RFQ_ERR_ALIGNMENT
    bad = rfq._KV(0, 2, 64, 16, 3, 16, None, 16, 16)
    assert lib.rfq_kv_read(ref(bad), 16, 3, 16, 16, 1, None) == rfq.RFQ_ERR_INVALID_ARG
    bad = rfq._KV(0, 2, 64, 16, 3, 16, 16, 20, 16)
    assert lib.rfq_kv_read(ref(bad), 16, 3, 16, 16, 1, None) == rfq.RFQ_ERR_ALIGNMENT


def test_attention_checks(lib):
    from paper_2608_26581_gb300 import rfq
    kv = rfq._KV(0, 2, 64, 16, 3, 16, 16, 16, 16)
    good = [16, 256, 64, 3, 4, None, 16, 3, ctypes.byref(kv), 16, 4, 0.125, 0, 16, 16, 16, None]

    def call(i, v):
        a = list(good)
        a[i] = v
        return lib.rfq_kv_attention(*a)
    for i in (0, 6, 8, 9, 13, 15):
        assert call(i, None) == rfq.RFQ_ERR_INVALID_ARG
    assert call(11, float("nan")) == rfq.RFQ_ERR_INVALID_ARG
    for i, v in ((3, -1), (3, 2), (4, 0), (4, 3), (7, -1), (10, 0), (10, 2 ** 27), (12, -1), (1, -8)):
        assert call(i, v) == rfq.RFQ_ERR_SHAPE
    for i, v in ((0, 24), (13, 8), (15, 4), (1, 252), (6, 18), (14, 18)):
        assert call(i, v) == rfq.RFQ_ERR_ALIGNMENT
    assert lib.rfq_kv_attention_workspace_bytes(4, 96) == 0 and lib.rfq_kv_attention_workspace_bytes(0, 64) == 0


def test_matvec_checks(lib):
    from paper_2608_26581_gb300 import rfq
    qt = lambda *a: ctypes.byref(rfq._QT(*a))  # noqa: E731
    ok = (0, 1, 64, 128, 16, 16)
    assert lib.rfq_matvec(16, 128, 1, None, 16, 0, None) == rfq.RFQ_ERR_INVALID_ARG
    assert lib.rfq_matvec(16, 128, 1, qt(*ok), 16, 3, None) == rfq.RFQ_ERR_INVALID_ARG
    assert lib.rfq_matvec(None, 128, 1, qt(*ok), 16, 0, None) == rfq.RFQ_ERR_INVALID_ARG
    assert lib.rfq_matvec(16, 128, 33, qt(*ok), 16, 0, None) == rfq.RFQ_ERR_SHAPE
    assert lib.rfq_matvec(16, 128, -1, qt(*ok), 16, 0, None) == rfq.RFQ_ERR_SHAPE
    assert lib.rfq_matvec(16, 128, 1, qt(0, 1, 64, 96, 16, 16), 16, 0, None) == rfq.RFQ_ERR_SHAPE
    assert lib.rfq_matvec(16, 128, 1, qt(0, 1, 2 ** 21 + 1, 128, 16, 16), 16, 0, None) == rfq.RFQ_ERR_SHAPE
    assert lib.rfq_matvec(16, 128, 1, qt(3, 1, 64, 128, 16, 16), 16, 0, None) == rfq.RFQ_ERR_UNSUPPORTED
    assert lib.rfq_matvec(16, 124, 1, qt(*ok), 16, 0, None) == rfq.RFQ_ERR_ALIGNMENT
    assert lib.rfq_matvec(8, 128, 1, qt(*ok), 16, 0, None) == rfq.RFQ_ERR_ALIGNMENT
