"""rfq_kv_attention for whole prompts: thousands of new tokens a request, many
tiles of 128 rows, every one with its own last key."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from paper_2608_26581_gb300.synth import bf16_bits_to_f32
from test_gpu_kv_attention import FMTS, Case, check

pytestmark = pytest.mark.gpu


def attention(c, window):
    """Softmax attention in 64 bits, a key head at a time."""
    q = torch.from_numpy(bf16_bits_to_f32(c.qb)).to(DEV).double()
    o, lse = torch.zeros_like(q), torch.full(q.shape[:2], -float("inf"), dtype=torch.float64, device=DEV)
    for r, (k, v) in enumerate(zip(c.keys, c.values)):
        rows, n, L = slice(c.start[r], c.start[r + 1]), c.new[r], c.lens[r]
        pos = torch.arange(L - n, L, device=DEV)[:, None]
        key = torch.arange(L, device=DEV)[None]
        hide = (key > pos) | ((key <= pos - window) if window else False)
        for h in range(c.H):
            heads = slice(h * c.G, (h + 1) * c.G)
            kh, vh = (torch.from_numpy(np.ascontiguousarray(x[:, h])).to(DEV) for x in (k, v))
            s = torch.einsum("tgd,kd->tgk", q[rows, heads], kh) * c.D ** -0.5
            s = s.masked_fill(hide[:, None], -float("inf"))
            z = torch.logsumexp(s, -1)
            lse[rows, heads] = z
            o[rows, heads] = torch.einsum("tgk,kd->tgd", torch.exp(s - z.clamp_min(-1e300)[..., None]), vh)
    return o.cpu().numpy(), lse.cpu().numpy()


@FMTS
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 700])
def test_prompts(fmt, D, window):
    """One behind cached tokens, one from the start, one token beside them."""
    c = Case(fmt, D, 2, 4, 64, [3500, 1111, 900], new=[3001, 1111, 1], seed=D + window)
    check(*c.run(window=window), *attention(c, window), c.vmax)
