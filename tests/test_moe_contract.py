"""What the header says of the entry points around a mixture-of-experts block,
without a GPU: sizes that are taken and refused, launches of unusual calls."""
import ctypes
import re

import pytest
import torch

from fake_kernels import FakeKernels
from paper_2608_26581_gb300 import rfq


# lengths of rows: all short ones, a spread of the others, and those at which a kernel changes
LENGTHS = [*range(1, 1100), *range(1100, 16385, 61), 2048, 2049, 2560, 2561, 4096, 4097, 4104, 5120, 5121, 5128, 8192, 8193, 8200, 12288, 12289, 12296, 16383, 16384]


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeKernels(tmp_path_factory.mktemp("fake"))


def test_rows_only_where_the_sort_takes_the_sizes(fake):
    """rfq_moe_rows: -1 exactly where rfq_moe_sort gives RFQ_ERR_SHAPE, else rows
    that fit 31 bits."""
    most = 2 ** 31 - 1
    for top_k, experts, align in ((8, 256, 4096), (1, 1, 1), (1, 256, 4096), (32, 256, 128), (8, 128, 1), (3, 5, 7)):
        border = (most - experts * align) // top_k
        for tokens in (0, 1, border - 1, border, border + 1, most // top_k, most // top_k + 1):
            rows = fake.lib.rfq_moe_rows(tokens, top_k, experts, align)
            status = fake.lib.rfq_moe_sort(256, tokens, top_k, experts, align, 256, 256, 256, max(rows, 0), 256, None)
            assert status == (rfq.RFQ_ERR_SHAPE if rows < 0 else rfq.RFQ_OK), (tokens, top_k, experts, align)
            assert rows <= most and (rows >= 0) == (tokens <= border)


def test_strides_along_one_element(fake):
    """A stride between tokens where there is one token, or between heads where
    there is one head, changes nothing: the same kernels, launched the same way."""
    qt = lambda: ctypes.byref(rfq._QT(0, 1, 24, 128, 256, 256))  # noqa: E731
    # (call, arguments with odd strides, which strides those are)
    norm = lambda t, h: (t, h, 256, t, h)  # noqa: E731
    cases = []
    for tokens, heads, odd in ((700, 1, (128, 131)), (1, 40, (5121, 128)), (1, 1, (129, 131)), (1, 1, (-1, -1))):
        for dtype in (0, 1):
            args = lambda t, h: (256, *norm(t, h), dtype, tokens, heads, 128, 0, 1e-6, 256, 256, 0, 256, 256, None)  # noqa: E731
            even = (odd[0] if tokens > 1 else 0, odd[1] if heads > 1 else 0)
            cases.append(("rfq_norm", args(*odd), args(*even)))
            args = lambda t, h: (256, *norm(t, h), 256, t, h, dtype, tokens, heads, 128, 0, 256, 256, 256, 0, 256, 256, 256, None)  # noqa: E731
            cases.append(("rfq_norm_grad", args(*odd), args(*even)))
    for dtype in (0, 1):
        for row in (129, -1):
            cases += [("rfq_route", *((256, r, dtype, 1, 128, 8, 1, 256, 256, None) for r in (row, 0))),
                      ("rfq_route_grad", *((256, r, dtype, 1, 128, 8, 1, 256, 256, 256, r, None) for r in (row, 0))),
                      ("rfq_moe_gather", *((256, r, dtype, 1, 128, 256, 8, 256, 256, 24, None) for r in (row, 0))),
                      ("rfq_moe_combine", *((256, dtype, 24, 128, 256, 256, 1, 8, 256, r, None) for r in (row, 0))),
                      ("rfq_moe_combine_grad", *((256, r, 256, dtype, 24, 128, 256, 256, 256, 1, 8, 256, 256, None) for r in (row, 0)))]
    cases += [("rfq_moe_quantize", *((256, r, 1, 256, 8, 256, qt(), qt(), None) for r in (row, 0))) for row in (129, -1)]
    for f, odd, even in cases:
        want = fake.call(f, *even)
        assert want[0] == rfq.RFQ_OK and want[1]
        assert fake.call(f, *odd) == want, (f, odd)


def test_binding_refuses_sizes_past_31_bits():
    """A size that C's int32 does not hold is refused, not taken modulo 2^32."""
    far = 2 ** 32
    new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="meta")  # noqa: E731
    i32 = lambda *s: new(*s, t=torch.int32)  # noqa: E731
    wide, few, ws = new(1, far + 128), new(3, 8), i32(64)
    q = rfq.QTensor(0, 1, 8, 128, new(512, t=torch.uint8), new(512, t=torch.uint8))
    calls = [lambda: rfq.rfq_norm(wide, wide), lambda: rfq.rfq_norm(new(1, far + 4, 8), new(1, far + 4, 8)),
             lambda: rfq.rfq_norm_grad(wide, wide, new(1), wide, mean=new(1)),
             lambda: rfq.rfq_norm_grad(new(1, far + 4, 8), new(1, far + 4, 8), new(far + 4), new(1, far + 4, 8)),
             lambda: rfq.rfq_route(wide, i32(1, 8), new(1, 8)), lambda: rfq.rfq_route(new(1, 8), i32(1, far + 2), new(1, far + 2)),
             lambda: rfq.rfq_route_grad(wide, i32(1, 8), new(1, 8), wide),
             lambda: rfq.rfq_moe_sort(i32(1, far + 2), i32(9), i32(1, far + 2), i32(16), ws), lambda: rfq.rfq_moe_sort(i32(3, 2), i32(far + 9), i32(3, 2), i32(16), ws),
             lambda: rfq.rfq_moe_sort(i32(3, 2), i32(9), i32(3, 2), i32(16), ws, align=far + 1), lambda: rfq.rfq_moe_sort(i32(3, 2), i32(9), i32(3, 2), i32(16), ws, align=1 - far),
             lambda: rfq.rfq_moe_gather(wide, i32(1, 2), new(2, far + 128)), lambda: rfq.rfq_moe_gather(few, i32(3, far + 2), few),
             lambda: rfq.rfq_moe_combine(new(2, far + 128), i32(1, 2), wide), lambda: rfq.rfq_moe_combine(few, i32(3, far + 2), few),
             lambda: rfq.rfq_moe_combine_grad(wide, new(2, far + 128), i32(1, 2), new(1, 2), new(2, far + 128), new(1, 2)),
             lambda: rfq.rfq_moe_combine_grad(few, few, i32(3, far + 2), new(3, far + 2), few, new(3, far + 2)),
             lambda: rfq.rfq_moe_quantize(new(3, 128, t=torch.bfloat16), i32(3, far + 2), q)]
    for i, f in enumerate(calls):
        with pytest.raises(rfq.RFQError) as e:
            f()
        assert e.value.status == rfq.RFQ_ERR_SHAPE, i
    assert rfq.rfq_norm_grad_workspace_bytes(far + 128) == 0
    for sizes in ((2 ** 64 + 4, 2, 8, 1), (4, far + 2, 8, 1), (4, 2, far + 8, 1), (4, 2, 8, far + 1), (4, 2, 8, 1 - far)):
        with pytest.raises(ValueError):
            rfq.rfq_moe_rows(*sizes)


def test_results_whose_rows_overlap(fake):
    """Several rows of a result in one place are refused (inputs may share rows)."""
    for t, h in ((0, 64), (63, 64), (256, 0), (256, 63)):
        for x in ((256, 64), (0, 64), (256, 0), (0, 0)):
            assert fake.call("rfq_norm", 256, *x, 256, t, h, 1, 3, 4, 64, 0, 1e-6, None, None, 0, None, None, None) == (rfq.RFQ_ERR_SHAPE, [])
            assert fake.call("rfq_norm", 256, *x, 256, 256, 64, 1, 3, 4, 64, 0, 1e-6, None, None, 0, None, None, None)[0] == rfq.RFQ_OK
            assert fake.call("rfq_norm_grad", 256, *x, 256, *x, 256, t, h, 1, 3, 4, 64, 0, 256, 256, None, 0, None, None, None, None) == (rfq.RFQ_ERR_SHAPE, [])
            assert fake.call("rfq_norm_grad", 256, *x, 256, *x, 256, 256, 64, 1, 3, 4, 64, 0, 256, 256, None, 0, None, None, None, None)[0] == rfq.RFQ_OK
    # heads before tokens
    assert fake.call("rfq_norm", 256, 64, 192, 256, 64, 192, 1, 3, 4, 64, 0, 1e-6, None, None, 0, None, None, None)[0] == rfq.RFQ_OK
    for row, status in ((0, rfq.RFQ_ERR_SHAPE), (127, rfq.RFQ_ERR_SHAPE), (128, rfq.RFQ_OK)):
        assert fake.call("rfq_route_grad", 256, 0, 0, 3, 128, 8, 1, 256, 256, 256, row, None)[0] == status
        assert fake.call("rfq_moe_combine", 256, 1, 24, 128, 256, 256, 3, 8, 256, row, None)[0] == status
    assert fake.call("rfq_moe_gather", 256, 0, 1, 3, 128, 256, 8, 256, 256, 24, None)[0] == rfq.RFQ_OK


def test_every_norm_kernel_is_reached(fake):
    """Some length and stride launches each kernel of the norms that is compiled,
    and the threads of a row hold all of its chunks."""
    compiled = {k for k in fake.kernels() if "norm_kernel" in k or "norm_grad_kernel" in k or "norm_sum_kernel" in k}
    start, n = fake.lib.fake_launched(), fake.lib.fake_launches()
    made = []                                # (dim, whether rows are narrow) of each launch
    for dim in LENGTHS:
        for dtype, words in ((0, 4), (1, 8)):
            for stride in {-(-dim // words) * words, -(-dim // words) * words + 1}:
                narrow = (stride | dim) % words != 0
                assert fake.lib.rfq_norm(256, stride, 0, 256, stride, 0, dtype, 2, 1, dim, 0, 1e-6, 256, 256, 0, 256, 256, None) == rfq.RFQ_OK
                assert fake.lib.rfq_norm_grad(256, stride, 0, 256, stride, 0, 256, stride, 0, dtype, 2, 1, dim, 0, 256, 256, 256, 0, 256, 256, 256,
                                              None) == rfq.RFQ_OK
                made += [(dim, dtype, narrow)] * 3
    reached = [fake.lib.fake_launched_kernel(start + i).decode() for i in range(len(made))]
    assert compiled == set(reached), sorted(compiled - set(reached))
    v = (ctypes.c_uint * 6)()
    for i, (kernel, (dim, dtype, narrow)) in enumerate(zip(reached, made)):
        split = re.search(r"SplitI(?:f|14__nv_bfloat16)Li(\d+)ELi(\d+)ELi(\d+)E", kernel)
        if split:
            vec, chunks, lanes = map(int, split.groups())
            fake.lib.fake_launch(n + i, v)
            assert vec == (1 + dtype if narrow else 4 + 4 * dtype)
            assert (v[3] if lanes > 32 else lanes) * chunks * vec >= dim, (kernel, dim)


def test_workspace_of_the_norms_gradient(fake):
    """Rows enough for every block: the blocks' partial sums fit the workspace for
    each length, wide and narrow, and fill it exactly for some of each; a block's
    shared memory is within what an SM's blocks have."""
    launch = (ctypes.c_uint * 6)()
    for device in (0, 1):
        fake.device(device)
        full = set()
        for dim in LENGTHS:
            padded, have = -(-dim // 4) * 4, fake.lib.rfq_norm_grad_workspace_bytes(dim)
            for dtype, words in ((0, 4), (1, 8)):
                for stride in {-(-dim // words) * words, dim + 1 - dim % 2}:
                    n = fake.lib.fake_launches()
                    assert fake.lib.rfq_norm_grad(256, stride, 0, 256, stride, 0, 256, stride, 0, dtype, 2 ** 20, 1, dim, 0, 256, 256, 256, 0, 256, 256, 256,
                                                  None) == rfq.RFQ_OK
                    assert fake.lib.fake_launches() == n + 2
                    fake.lib.fake_launch(n, launch)
                    blocks, threads, smem = launch[0], launch[3], launch[5]
                    assert blocks * 2 * padded * 4 <= have, (dim, dtype, stride)
                    # (512 static bytes beside the dynamic ones; 228 KB an SM)
                    assert threads <= 1024 and smem <= 200 * 1024
                    if blocks * 2 * padded * 4 == have:
                        full.add((dim > 8192, 256 < dim <= 512, (stride | dim) % words != 0))
        # (wide rows of 257 to 512 elements take a warp each, and two blocks an SM where the workspace has ten)
        assert {(False, False, False), (False, False, True), (False, True, True), (True, False, False), (True, False, True)} <= full
    fake.device(0)
