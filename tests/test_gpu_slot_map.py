"""rfq_slot_map against a request-by-request allocator: whole numbers, so
every output is equal."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import DEV, guarded_empty, guarded_full
from paper_2608_26581_gb300 import rfq

pytestmark = pytest.mark.gpu
I32 = torch.int32


def _dev(a, dtype=I32):
    t = guarded_empty((max(1, len(a)),), dtype)[:len(a)]
    t.copy_(torch.tensor(np.asarray(a)).to(dtype))
    return t


def _run(cached, added, page, table, free, count, tokens, alias=False):
    R, width = table.shape
    tb = guarded_empty((max(R, 1), width), I32)[:R]
    tb.copy_(torch.from_numpy(table))
    fr, cnt = _dev(free), _dev([count])
    ca = _dev(cached)
    out, ln = (cnt, ca) if alias else (guarded_full((1,), -7, I32), guarded_full((max(R, 1),), -7, I32)[:R])
    st = guarded_full((R + 1,), -7, I32)
    sl, po = guarded_full((max(tokens, 1),), -7, torch.int64)[:tokens], guarded_full((max(tokens, 1),), -7, I32)[:tokens]
    ws = torch.zeros(64, dtype=I32, device=DEV)
    rfq.rfq_slot_map(ca, _dev(added), page, tb, fr, cnt, out, ln, st, sl, po, ws)
    bad = rfq.rfq_workspace_status(ws) == rfq.RFQ_ERR_SHAPE
    return [t.cpu().numpy() for t in (tb, fr, out, ln, st, sl, po)] + [bad]


def _check(cached, added, page, width, free, count, tokens, seed=0, alias=False):
    rng = np.random.default_rng(seed)
    R = len(cached)
    table = rng.permutation(R * width + 7)[:R * width].reshape(R, width).astype(np.int32)
    want = ref.slot_map(cached, added, page, table, np.asarray(free, np.int32), count, tokens)
    got = _run(cached, added, page, table, free, count, tokens, alias)
    for g, w, name in zip(got, want, ("table", "free", "count", "lengths", "start", "slots", "positions", "bad")):
        np.testing.assert_array_equal(np.asarray(g).reshape(-1), np.asarray(w).reshape(-1), err_msg=name)


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("R", [1, 2, 31, 33, 1000, 1025, 8192])
def test_random_steps(R, alias):
    rng = np.random.default_rng(R)
    page, width = 16, 40
    cached = rng.integers(0, 500, R)
    added = np.where(rng.random(R) < 0.2, -rng.integers(0, 600, R), rng.integers(0, 4 if R > 100 else 100, R))
    free = list(rng.permutation(10 ** 6)[:R * width]) + [0] * (R * width)
    total = int(np.maximum(added, 0).sum())
    _check(cached.tolist(), added.tolist(), page, width, free, R * width, total + 3, seed=R, alias=alias)


@pytest.mark.parametrize("count", [0, 1, 5, 6, 7])
def test_pages_run_out(count):
    """Requests are served until one does not fit; later ones that want no
    page still are, and pages given back in the same step are used."""
    _check([0, 16, 30, 5, 15, 64], [32, 1, 1, 200, 2, -20], 16, 20, list(range(100, 110)), count, 260)


@pytest.mark.parametrize("page", [1, 16, 48, 4096])
def test_page_sizes(page):
    _check([0, page - 1, page, 3 * page + 1], [2 * page + 1, 1, 1, -2 * page], page, 6, list(range(50, 70)), 20, 2 * page + 9)


def test_long_prompt_spread_over_ctas():
    _check([100, 0, 7], [1, 20000, 1], 16, 1300, list(range(2000)), 2000, 20002)


def test_no_requests_and_no_tokens():
    _check([], [], 16, 4, [1, 2, 3], 2, 5)
    _check([3, 16], [0, -16], 16, 4, [1, 2, 3], 1, 0)


def test_too_few_token_rows_or_table_columns_set_the_status():
    _check([0, 4], [9, 3], 16, 4, [1, 2, 3], 3, 10)         # 12 tokens, 10 rows
    _check([0, 60, 2], [9, 10, 3], 16, 4, [1, 2, 3], 3, 22)  # 70 tokens do not fit four pages
    _check([-5, 2], [9, 3], 16, 4, [1, 2, 3], 3, 12)         # a negative length
    _check([64, 2], [-64, 3], 16, 4, [1, 2, 3], 2, 3)        # four pages given back, room for one
