"""rfq_kv_attention where a few keys hold nearly all of a row's weight and their
values are nothing (an attention sink): the output is made of the small
weights, which have to keep their accuracy beside the large ones."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import DEV
from paper_2608_26581_gb300 import rfq
from paper_2608_26581_gb300.synth import bf16_bits_to_f32, f32_to_bf16_bits
from test_gpu_kv_attention import FMTS, Case, bits_to_dev

pytestmark = pytest.mark.gpu
EVERY = 32                                # one sink in each such run of keys


def fill(c, octaves):
    """Keys of c that lie 2^octaves below the sinks among them, up to a tenth of
    an octave, and values near one, zero at the sinks; the scale that makes it so."""
    rng = np.random.default_rng(int(octaves * 10))
    slots = [int(c.table[r, j // c.page]) * c.page + j % c.page for r, n in enumerate(c.lens) for j in range(n)]
    where = np.concatenate([np.arange(n) for n in c.lens]) % EVERY == 5
    T, H, D = len(slots), c.H, c.D
    k = 0.05 * rng.standard_normal((T, H, D))
    v = 1 + 0.3 * rng.standard_normal((T, H, D))
    k[..., 0] = 0
    k[where], v[where] = 0, 0
    k[where, :, 0] = 6
    s = torch.tensor(slots, device=DEV)
    rfq.rfq_kv_append(bits_to_dev(f32_to_bf16_bits(k.astype(np.float32))), bits_to_dev(f32_to_bf16_bits(v.astype(np.float32))), s, c.cache)
    ko, vo = torch.empty(T, H, D, device=DEV), torch.empty(T, H, D, device=DEV)
    rfq.rfq_kv_read(c.cache, s, ko, vo)
    cut = np.cumsum(c.lens)[:-1]
    c.keys, c.values = np.split(ko.double().cpu().numpy(), cut), np.split(vo.double().cpu().numpy(), cut)
    q = 0.25 * rng.standard_normal(c.qb.shape)
    q[..., 0] = 4
    c.qb = f32_to_bf16_bits(q.astype(np.float32))
    return octaves * np.log(2) / 24


def check(c, scale):
    """A weight is rounded to f16: by 2^-11 of itself, or by 2^-25 of the unit
    2^m it is held in where f16 has no more bits.  The unit lies 2^7 or more
    below the largest weight of those that are summed with it, a sink's, so the
    second part is at most 2^-32 of a sink's weight a key.  Beside them bf16's
    rounding of the output and the fp32 sums, 2^-16 of the sum of |w v|."""
    o, lse = c.run(scale=scale)
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    q = bf16_bits_to_f32(c.qb).astype(np.float64)
    want, want_lse = ref.attention(q, c.keys, c.values, c.start, c.lens, scale, 0)
    mag = ref.attention(q, c.keys, [np.abs(v) for v in c.values], c.start, c.lens, scale, 0)[0]
    for r, (k, v) in enumerate(zip(c.keys, c.values)):
        rows = slice(c.start[r], c.start[r + 1])
        for h in range(c.H):
            heads = slice(h * c.G, (h + 1) * c.G)
            sink = np.exp(q[rows, heads] @ k[5, h] * scale - want_lse[rows, heads])
            bound = 2.0 ** -8 * np.abs(want[rows, heads]) + (2.0 ** -11 + 2.0 ** -16) * mag[rows, heads] + \
                2.0 ** -32 * sink[..., None] * np.abs(v[:, h]).sum(0)
            err = np.abs(o[rows, heads] - want[rows, heads])
            assert (err <= bound).all(), f"worst {np.max(err / bound):.3f} of the bound"
    assert (np.abs(lse - want_lse) <= 2.0 ** -17 * (1 + np.abs(want_lse))).all()


@FMTS
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 4, 30])
@pytest.mark.parametrize("octaves", [12, 16, 20, 23.4, 25.5])
def test_small_weights_beside_sinks(fmt, D, new, octaves):
    """Of one token, of several, and of enough for the tiles of 128 rows."""
    c = Case(fmt, D, 2, 4, 16, [700, 64, 333], new=[new] * 3, seed=1)
    check(c, fill(c, octaves))


@FMTS
def test_one_sink_in_a_long_request(fmt):
    """The usual place, the first keys: what is summed with them is small."""
    for new in (1, 40):
        c = Case(fmt, 64, 2, 4, 64, [9000], new=[new], seed=2)
        scale = fill(c, 22)
        k, v = (torch.from_numpy(x[0].astype(np.float32)).to(DEV) for x in (c.keys, c.values))
        slots = torch.tensor([int(c.table[0, j // 64]) * 64 + j % 64 for j in range(9000)], device=DEV)
        later = torch.arange(9000, device=DEV) % EVERY == 5
        later[5] = False
        k[later], v[later] = 0, 1
        rfq.rfq_kv_append(k.bfloat16(), v.bfloat16(), slots, c.cache)
        rfq.rfq_kv_read(c.cache, slots, k, v)
        c.keys, c.values = [k.double().cpu().numpy()], [v.double().cpu().numpy()]
        check(c, scale)
