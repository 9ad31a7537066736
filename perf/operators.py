"""Cases for the operators of one attention step on a 4-bit cache, and the
plain forms their results are held against.

  slots    block tables, slot maps and positions from the requests' lengths
  rope     rotary positions with several axes, and their gradient
  append   keys and values quantized into the paged 4-bit cache, and read back
  attn     attention over the paged 4-bit cache
  matvec   y = x W~^T for a few tokens, W~ in 4 bits with group scales

``run`` computes a case in elementary torch operations in 32 bits, or through
the library's entry points where ``own`` is set.  The layouts of the cache and
of quantized weights are those that include/rfq.h documents.
"""
import math
import random

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # a serving step of a large batch: almost every request adds one token, some end, some begin with a prompt
        {"name": "slots decode", "op": "slots", "requests": 256, "page": 16, "longest": 4096, "prompt": 0, "seqs": 1},
        # prompts of a batch enter at once, one of them long
        {"name": "slots prompts", "op": "slots", "requests": 37, "page": 64, "longest": 16384, "prompt": 8192, "seqs": 2},
        # queries of one Wan2.2-14B DiT layer over a whole clip: three axes, neighbouring dimensions paired
        {"name": "rope video", "op": "rope", "tokens": 32760, "heads": 40, "row": 40, "dim": 128, "rot": 128, "axes": 3, "pair": 1,
         "inverse": False, "dtype": "bf16"},
        # gradient of queries and keys in the packed projection of a Qwen3-VL layer
        {"name": "rope gradient", "op": "rope", "tokens": 4096, "heads": 40, "row": 48, "dim": 128, "rot": 128, "axes": 3, "pair": 0,
         "inverse": True, "dtype": "f32"},
        # one new token for each of a batch of requests
        {"name": "append decode", "op": "append", "tokens": 61, "heads": 8, "dim": 128, "page": 16, "fmt": "mxfp4"},
        # the keys and values of long prompts
        {"name": "append prompt", "op": "append", "tokens": 16384, "heads": 8, "dim": 128, "page": 64, "fmt": "hif4"},
        # one user, a short conversation: latency
        {"name": "attn one", "op": "attn", "requests": 1, "least": 777, "longest": 777, "new": 0, "heads": 32, "kv": 8, "dim": 128, "page": 16,
         "window": 0, "fmt": "mxfp4"},
        # ordinary serving: ragged lengths, Qwen3-VL-30B-A3B's heads
        {"name": "attn batch", "op": "attn", "requests": 64, "least": 0, "longest": 8192, "new": 0, "heads": 32, "kv": 4, "dim": 128, "page": 64,
         "window": 0, "fmt": "mxfp4"},
        # long contexts, Qwen3-VL-8B's heads
        {"name": "attn long", "op": "attn", "requests": 8, "least": 98304, "longest": 131072, "new": 0, "heads": 32, "kv": 8, "dim": 128,
         "page": 64, "window": 0, "fmt": "hif4"},
        # chunks of new prompt tokens over what is cached
        {"name": "attn chunk", "op": "attn", "requests": 5, "least": 300, "longest": 8192, "new": 256, "heads": 32, "kv": 8, "dim": 128,
         "page": 32, "window": 0, "fmt": "mxfp4"},
        # one token through the gate/up projection of a Qwen3-VL-8B layer
        {"name": "matvec one", "op": "matvec", "rows": 1, "k": 4096, "n": 24576, "fmt": "mxfp4", "scales": "mma", "out": "bf16"},
        # a small batch through its down projection
        {"name": "matvec batch", "op": "matvec", "rows": 13, "k": 12288, "n": 4096, "fmt": "hif4", "scales": "mma", "out": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["slots", "rope", "append", "attn", "attn", "matvec", "matvec"])
    if op == "slots":
        prompt = rng.choice([0, _log(rng, 2, 8192)])
        return {"op": op, "requests": _log(rng, 1, 512), "page": 16 * rng.choice([1, 2, 3, 4, 8]), "longest": _log(rng, 64, 16384),
                "prompt": prompt, "seqs": rng.choice([1, 2])}
    if op == "rope":
        dim = rng.choice([64, 80, 128, 128, 128])
        rot = rng.choice([dim, dim, dim // 2])
        heads, dtype = rng.randint(1, 40), rng.choice(["bf16", "f32"])
        return {"op": op, "tokens": _log(rng, 1, 16384 if dtype == "bf16" else 2048), "heads": heads, "row": heads + rng.choice([0, 0, 8]), "dim": dim, "rot": rot,
                "axes": rng.choice([1, 3]), "pair": rng.choice([0, 1]), "inverse": rng.random() < 0.5, "dtype": dtype}
    if op == "append":
        return {"op": op, "tokens": _log(rng, 1, 16384), "heads": rng.choice([1, 2, 4, 8, 8]), "dim": rng.choice([64, 128, 128]),
                "page": 16 * rng.choice([1, 2, 3, 4, 8]), "fmt": rng.choice(["mxfp4", "hif4"])}
    if op == "attn":
        kv = rng.choice([1, 2, 4, 8, 8])
        requests = _log(rng, 1, 128)
        longest = _log(rng, 16, min(65536, 2 ** 22 // (requests * kv)))
        new = rng.choice([0, 0, 0, _log(rng, 2, 64)])
        return {"op": op, "requests": requests, "least": rng.choice([0, 1, longest // 2]), "longest": longest, "new": new,
                "heads": kv * rng.choice([1, 3, 4, 5, 8, 8]), "kv": kv, "dim": rng.choice([64, 128, 128]), "page": 16 * rng.choice([1, 2, 3, 4, 8]),
                "window": rng.choice([0, 0, 0, _log(rng, 16, 4096)]), "fmt": rng.choice(["mxfp4", "hif4"])}
    fmt = rng.choice(["mxfp4", "hif4"])
    scales = rng.choice(["mma", "rows"])
    step = 64 if fmt == "hif4" else 128 if scales == "mma" else 32
    return {"op": op, "rows": rng.choice([1, 1, 2, rng.randint(3, 32)]), "k": max(step, _log(rng, 256, 12288) // step * step),
            "n": _log(rng, 64, 13824), "fmt": fmt, "scales": scales, "out": rng.choice(["bf16", "f32"])}


# ---------------------------------------------------------------- formats

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _quant_mxfp4(x):
    """fp32 [..., n] (n % 32 == 0) -> codes int32 [..., n], E8M0 bytes int32 [..., n / 32]."""
    b = x.unflatten(-1, (-1, 32))
    e = ((b.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp_min(0)
    s = torch.where(e > 0, e << 23, torch.full_like(e, 0x400000)).view(torch.float32)
    y = b.abs() / s.unsqueeze(-1)
    # the grid of E2M1: steps of 1/2 below 2, of 1 below 4, of 2 above; ties to even
    k = torch.where(y < 2, (y * 2).round(), torch.where(y < 4, y.round() + 2, (y / 2).round() + 4)).clamp_max(7).int()
    return (k + 8 * torch.signbit(b).int()).flatten(-2), e


def _hif4_scale(meta):
    return (((((meta >> 2) & 63) + 79) << 23) | ((meta & 3) << 21)).view(torch.float32)


def _quant_hif4(x):
    """fp32 [..., n] (n % 64 == 0) -> codes int32 [..., n], metadata words int32 [..., n / 64]."""
    b = x.unflatten(-1, (-1, 64))
    a = b.abs().amax(-1)
    sevens = 7 * _hif4_scale(torch.arange(256, device=x.device, dtype=torch.int32))
    byte = torch.searchsorted(sevens, a.contiguous()).clamp_max(255).int()
    s = _hif4_scale(byte)
    g = b.unflatten(-1, (16, 4))
    ag = g.abs().amax(-1)
    t = (ag > 1.75 * s.unsqueeze(-1)).int() + (ag > 3.5 * s.unsqueeze(-1)).int()
    e8 = (t.unflatten(-1, (8, 2)).amax(-1) == 2).int()
    e16 = (t - e8.repeat_interleave(2, -1)).clamp_min(0)
    ex = e16 + e8.repeat_interleave(2, -1)
    step = 0.25 * s.unsqueeze(-1) * (1 << ex).float()
    k = (g.abs() / step.unsqueeze(-1)).round().clamp_max(7).int()
    codes = (k + 8 * torch.signbit(g).int()).flatten(-3)
    bits8 = (e8 << torch.arange(8, 16, device=x.device, dtype=torch.int32)).sum(-1, dtype=torch.int32)
    bits16 = (e16 << torch.arange(16, 32, device=x.device, dtype=torch.int32)).sum(-1, dtype=torch.int32)
    return codes, torch.where(a > 0, byte | bits8 | bits16, torch.zeros_like(byte))


def _values_mxfp4(codes, scales):
    """codes int32 [..., n], E8M0 bytes int32 [..., n / 32] -> fp32 values."""
    v = torch.tensor(E2M1 + [-a for a in E2M1], device=codes.device)[codes]
    s = torch.where(scales > 0, scales << 23, torch.full_like(scales, 0x400000)).view(torch.float32)
    return (v.unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _values_hif4(codes, meta):
    """codes int32 [..., n], metadata words int32 [..., n / 64] -> fp32 values."""
    k = torch.where(codes >= 8, 8 - codes, codes).float().unflatten(-1, (-1, 16, 4))
    i = torch.arange(16, device=codes.device, dtype=torch.int32)
    ex = ((meta.unsqueeze(-1) >> (8 + i // 2)) & 1) + ((meta.unsqueeze(-1) >> (16 + i)) & 1)
    step = 0.25 * _hif4_scale(meta).unsqueeze(-1) * (1 << ex).float()
    return (k * step.unsqueeze(-1)).flatten(-3)


def _pack(codes):
    """int32 codes [..., n] -> uint8 [..., n / 2], element 2j in the low nibble."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).to(torch.uint8)


def _unpack(b):
    b = b.int()
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


# ---------------------------------------------------------------- the cache
# codes and scales of one page and head hold page_size tokens:
#   K codes   [page][4][D/32][4] bytes: the 4-byte word of dimensions 32 b + 8 c .. + 7 of a token is word (c, b) of its row
#   V codes   [page/16][2][8][4][2][D/16] bytes: token 16 i + 8 h + 2 c + j, dimensions g D/8 .. at (i, h, g, c, j)
#   scales    MXFP4: [page][D/32] bytes; HiF4: [page][D/64] words of 4 bytes


def _store(x, fmt, value):
    """fp32 [pages, heads, page, D] -> codes uint8, scales uint8 as a cache holds them."""
    pages, heads, page, D = x.shape
    codes, sc = _quant_mxfp4(x) if fmt == "mxfp4" else _quant_hif4(x)
    c = _pack(codes)
    if value:
        c = c.view(pages, heads, page // 16, 2, 4, 2, 8, D // 16).permute(0, 1, 2, 3, 6, 4, 5, 7)
    else:
        c = c.view(pages, heads, page, D // 32, 4, 4).transpose(3, 4)
    sc = sc.to(torch.uint8) if fmt == "mxfp4" else sc.contiguous().view(torch.uint8)
    return c.reshape(pages, heads, page * D // 2).contiguous(), sc.reshape(pages, heads, -1).contiguous()


def _load(codes, scales, page, D, fmt, value):
    """codes uint8 [..., page D / 2], scales uint8 [..., n] of whole pages -> fp32 [..., page, D]."""
    if value:
        c = codes.unflatten(-1, (page // 16, 2, 8, 4, 2, D // 16))
        c = c.movedim(-4, -2).flatten(-6)
    else:
        c = codes.unflatten(-1, (page, 4, D // 32, 4)).transpose(-3, -2).flatten(-4)
    c = _unpack(c).unflatten(-1, (page, D))
    if fmt == "mxfp4":
        return _values_mxfp4(c, scales.int().unflatten(-1, (page, D // 32)))
    return _values_hif4(c, scales.contiguous().view(torch.int32).unflatten(-1, (page, D // 64)))


def _activations(g, shape):
    """fp32 values as a projection gives them (exact in bf16): a few channels stand out."""
    x = torch.randn(shape, generator=g, device=DEV)
    c = 1 + 15 * (torch.rand(shape[-2:], generator=g, device=DEV) < 0.02).float()
    return (x * c).bfloat16().float()


def _empty_cache(pages, heads, page, D, fmt):
    n = page * (D // 32 if fmt == "mxfp4" else D // 16)
    z = lambda m: torch.zeros(pages, heads, m, dtype=torch.uint8, device=DEV)  # noqa: E731
    return [z(page * D // 2), z(n), z(page * D // 2), z(n)]


def _handle(case, arrays):
    """The library's handle of a cache (its arrays, sizes and format), kept for the cache's life."""
    from paper_2608_26581_gb300 import rfq
    fmt = rfq.RFQ_FMT_MXFP4 if case["fmt"] == "mxfp4" else rfq.RFQ_FMT_HIF4
    heads = case["kv"] if "kv" in case else case["heads"]
    return rfq.KVCache(fmt, heads, case["dim"], case["page"], arrays[0].shape[0], *arrays)


# ---------------------------------------------------------------- prepare

def _lengths(case, seed):
    """Host lists of an attention case: cached tokens and new tokens of each request."""
    r, kinds = random.Random(seed * 7 + 1), random.Random(5)  # the new tokens are the case's own: its outputs have one shape
    lo, hi = case["least"], case["longest"]
    new = [kinds.randint(1, case["new"]) if case["new"] else 1 for _ in range(case["requests"])]
    lens = [lo if i % 7 == 5 else _log(r, max(1, lo), max(1, hi)) for i in range(case["requests"])]
    if case["requests"] > 1:
        lens[-1] = hi
    return lens, new


def _step(case, seed):
    """Host lists of a slots case: cached tokens of each request, and tokens that it adds (or, below zero, drops)."""
    r, kinds = random.Random(seed * 5 + 3), random.Random(3)  # what is added is the case's own: its outputs have one shape
    cached, added = [], []
    for _ in range(case["requests"]):
        c, a, kind = _log(r, 1, case["longest"]), case["seqs"], kinds.random()
        if case["prompt"] and kind < 0.5:
            c, a = r.choice([0, c]), _log(kinds, 1, case["prompt"])
        elif kind > 0.9:
            a = r.choice([-c, -min(c, 3), 0])
        cached.append(c)
        added.append(a)
    return cached, added


def prepare(case, seed):
    op = case["op"]
    g = _gen(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if op == "slots":
        page, R = case["page"], case["requests"]
        cached, added = _step(case, seed)
        pages = lambda n: -(-n // page)  # noqa: E731
        width = pages(case["longest"] + case["prompt"] + case["seqs"]) + 1
        used = sum(pages(c) for c in cached)
        need = sum(max(0, pages(c + a) - pages(c)) for c, a in zip(cached, added))
        count = need - (need // 5 if seed % 4 == 3 else 0)  # now and then the pages run out
        ids = torch.randperm(R * width, generator=g, device=DEV).int()
        table = torch.full((R, width), -1, dtype=torch.int32, device=DEV)
        have = i32([pages(c) for c in cached])
        at = torch.arange(width, device=DEV)[None] < have[:, None]
        table[at] = ids[:used]
        free = torch.full((R * width,), -1, dtype=torch.int32, device=DEV)
        free[:count] = ids[used:used + count]
        T = sum(max(0, a) for a in added) + 5  # a step's fixed capacity
        s = {"op": op, "page": page, "cached": i32(cached), "added": i32(added), "table": table, "free": free, "count": i32([count]),
             "count_out": i32([0]), "lengths": i32([0] * R), "start": i32([0] * (R + 1)),
             "slots": torch.zeros(T, dtype=torch.int64, device=DEV), "positions": torch.zeros(T, dtype=torch.int32, device=DEV)}
        if own:
            s["ws"] = torch.zeros(64, dtype=torch.int32, device=DEV)
        return s
    if op == "rope":
        T, D, P = case["tokens"], case["dim"], case["rot"] // 2
        x = _activations(g, (T, case["row"], D))
        x = x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        t = torch.arange(T, device=DEV)
        # (angles in 32 bits, as the plain form has them, hold fp32 outputs at low positions alone)
        far = 100000 if case["dtype"] == "bf16" else 1000
        if case["axes"] == 3:  # a clip of frames of 30 x 52 patches
            pos = torch.stack((t // 1560, t // 52 % 30, t % 52)) + torch.randint(0, far // 50 + 980, (1, 1), generator=g, device=DEV)
        else:
            pos = t[None] + torch.randint(0, far, (1, 1), generator=g, device=DEV)
        if case["pair"] == 1 and case["axes"] == 3:  # each axis has a run of pairs and its own frequencies
            n = [P - 2 * (P // 3), P // 3, P // 3]
            axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(n, device=DEV))
            f = torch.cat([10000.0 ** (-torch.arange(m, device=DEV, dtype=torch.float64) / max(1, m)) for m in n])
        else:  # one progression of frequencies, the axes in turn
            axis = torch.arange(P, device=DEV) % case["axes"]
            f = 1e6 ** (-torch.arange(P, device=DEV, dtype=torch.float64) / P)
        return {"op": op, "x": x[:, :case["heads"]], "pos": pos.int().contiguous(), "freq": f.float(), "axis": axis.int(), "pair": case["pair"],
                "inverse": case["inverse"], "out": torch.empty(T, case["heads"], D, dtype=x.dtype, device=DEV)}
    if op == "append":
        T, H, D, page = case["tokens"], case["heads"], case["dim"], case["page"]
        pages = T // page + 3
        kv = _activations(g, (T, 2 * H, D)).bfloat16()
        arrays = _empty_cache(pages, H, page, D, case["fmt"])
        slots = torch.randperm(pages * page, generator=g, device=DEV)[:T] if T < 256 else \
            (torch.randperm(pages, generator=g, device=DEV)[:, None] * page + torch.arange(page, device=DEV)).flatten()[:T].contiguous()
        s = {"op": op, "fmt": case["fmt"], "page": page, "k": kv[:, :H], "v": kv[:, H:], "slots": slots, "arrays": arrays,
             "ko": torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV), "vo": torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)}
        if own:
            s["cache"] = _handle(case, arrays)
        return s
    if op == "attn":
        lens, new = _lengths(case, seed)
        H, D, page, fmt, R = case["kv"], case["dim"], case["page"], case["fmt"], case["requests"]
        have = [-(-n // page) for n in lens]
        pages = sum(have) + 1
        some = min(pages, max(1, 2 ** 22 // (page * H * D)))  # pages of distinct values; the others repeat them
        which = torch.randint(0, some, (pages,), generator=g, device=DEV)
        arrays = []
        for value in (False, True):
            x = _activations(g, (some, page, H, D)).transpose(1, 2)
            arrays += [a[which] for a in _store(x, fmt, value)]
        ids = torch.randperm(pages, generator=g, device=DEV).int()
        table = torch.full((R, max(1, max(have))), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(table.shape[1], device=DEV)[None] < i32(have)[:, None]] = ids[:sum(have)]
        T = sum(new)
        q = torch.randn(T, case["heads"] + 2 * H, D, generator=g, device=DEV).bfloat16()[:, :case["heads"]]  # of a packed projection
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        s = {"op": op, "fmt": fmt, "page": page, "q": q, "arrays": arrays, "table": table, "lens": i32(lens),
             "start": i32(start) if case["new"] else None, "scale": D ** -0.5, "window": case["window"], "most": max(new),
             "out": torch.empty(T, case["heads"], D, dtype=torch.bfloat16, device=DEV),
             "lse": torch.empty(T, case["heads"], dtype=torch.float32, device=DEV)}
        if own:
            from paper_2608_26581_gb300 import rfq
            s["cache"] = _handle(case, arrays)
            s["ws"] = rfq.kv_attention_workspace(case["heads"], D)
        return s
    K, N, M = case["k"], case["n"], case["rows"]
    x = torch.randn(M, K, generator=g, device=DEV) * (1 + 49 * (torch.rand(K, generator=g, device=DEV) < 0.01).float())
    w = (torch.randn(N, K, generator=g, device=DEV) * 0.02).bfloat16().float()
    codes, sc = _quant_mxfp4(w) if case["fmt"] == "mxfp4" else _quant_hif4(w)
    codes, n128 = _pack(codes), -(-N // 128) * 128
    if case["scales"] == "rows":
        sc = sc.to(torch.uint8) if case["fmt"] == "mxfp4" else sc
    elif case["fmt"] == "mxfp4":  # atoms of 128 rows x 4 blocks, row m of an atom at (m % 32) 16 + (m / 32) 4
        p = torch.zeros(n128, K // 32, dtype=torch.uint8, device=DEV)
        p[:N] = sc.to(torch.uint8)
        sc = p.view(n128 // 128, 4, 32, K // 128, 4).permute(0, 3, 2, 1, 4)
    else:  # block-major, the rows of a block padded to 128
        p = torch.zeros(n128, K // 64, dtype=torch.int32, device=DEV)
        p[:N] = sc
        sc = p.t()
    sc = sc.contiguous().view(torch.uint8).flatten()
    s = {"op": op, "fmt": case["fmt"], "scales": case["scales"], "x": x.bfloat16(), "codes": codes, "sc": sc,
         "y": torch.empty(M, N, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device=DEV)}
    if own:
        from paper_2608_26581_gb300 import rfq
        s["w"] = rfq.QTensor(rfq.RFQ_FMT_MXFP4 if case["fmt"] == "mxfp4" else rfq.RFQ_FMT_HIF4,
                             rfq.RFQ_SCALE_MMA if case["scales"] == "mma" else rfq.RFQ_SCALE_ROWMAJOR, N, K, codes.flatten(), sc)
    return s


# ---------------------------------------------------------------- run

def run(s):
    if own:
        return _own(s)
    return {"slots": _plain_slots, "rope": _plain_rope, "append": _plain_append, "attn": _plain_attn, "matvec": _plain_matvec}[s["op"]](s)


def _own(s):
    from paper_2608_26581_gb300 import rfq
    if s["op"] == "slots":
        rfq.rfq_slot_map(s["cached"], s["added"], s["page"], s["table"], s["free"], s["count"], s["count_out"], s["lengths"], s["start"],
                         s["slots"], s["positions"], s["ws"])
        return {k: s[k] for k in ("table", "free", "count_out", "lengths", "start", "slots", "positions")}
    if s["op"] == "rope":
        rfq.rfq_rope(s["x"], s["out"], s["pos"], s["freq"], s["axis"], pairing=s["pair"], inverse=s["inverse"])
        return s["out"]
    if s["op"] == "append":
        rfq.rfq_kv_append(s["k"], s["v"], s["slots"], s["cache"])
        rfq.rfq_kv_read(s["cache"], s["slots"], s["ko"], s["vo"])
        return {"k": s["ko"], "v": s["vo"]}
    if s["op"] == "attn":
        rfq.rfq_kv_attention(s["q"], s["cache"], s["table"], s["lens"], s["out"], s["ws"], lse=s["lse"], q_start=s["start"], scale=s["scale"],
                             window=s["window"])
        return {"o": s["out"], "lse": s["lse"]}
    rfq.rfq_matvec(s["x"], s["w"], s["y"])
    return s["y"]


def _plain_slots(s):
    page, table, free = s["page"], s["table"], s["free"]
    cached, added = s["cached"].long(), s["added"].long()
    R, width = table.shape
    after = (cached + added).clamp_min(0)
    p0, p1 = (cached + page - 1) // page, (after + page - 1) // page
    fits = p1 <= width
    need = torch.where(fits, (p1 - p0).clamp_min(0), 0)
    back = (p0 - p1).clamp_min(0)
    j = torch.arange(width, device=table.device)[None]
    # pages given back go on top of the list, in the order of the requests and of their tables
    n1 = s["count"].long() + back.sum()
    to = s["count"].long() + (back.cumsum(0) - back)[:, None] + j - p1[:, None]
    gives = (j >= p1[:, None]) & (j < p0[:, None])
    spare = torch.cat((free, free[:1]))
    spare.scatter_(0, torch.where(gives, to, free.numel()).flatten(), table.flatten())
    free.copy_(spare[:-1])
    # pages are taken from the top, request by request, until one cannot be served
    upto = need.cumsum(0)
    served = fits & ((need == 0) | (upto <= n1))
    takes = (j >= p0[:, None]) & (j < p1[:, None]) & served[:, None]
    nth = (upto - need)[:, None] + j - p0[:, None]
    table.copy_(torch.where(takes, free[(n1 - 1 - nth).clamp(0, free.numel() - 1)], table))
    s["count_out"].copy_(n1 - torch.where(served, upto, 0).amax())
    s["lengths"].copy_(torch.where(served, after, cached))
    n = added.clamp_min(0)
    s["start"][1:] = n.cumsum(0)
    t = torch.arange(s["slots"].numel(), device=table.device)
    row = torch.searchsorted(s["start"][1:].long(), t, right=True)
    there = row < R
    row = row.clamp_max(R - 1)
    pos = cached[row] + t - s["start"][row]
    at = table[row, (pos // page).clamp(0, width - 1)].long() * page + pos % page
    s["slots"].copy_(torch.where(there & served[row], at, -1))
    s["positions"].copy_(torch.where(there, pos, 0))
    return {k: s[k] for k in ("table", "free", "count_out", "lengths", "start", "slots", "positions")}


def _plain_rope(s):
    x = s["x"].float()
    P = s["freq"].numel()
    angle = s["pos"][s["axis"].long()].t().float() * s["freq"]  # [T, P]
    c, sn = angle.cos()[:, None], angle.sin()[:, None]
    if s["inverse"]:
        sn = -sn
    if s["pair"] == 1:
        a, b = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
        r = torch.stack((a * c - b * sn, b * c + a * sn), -1).flatten(-2)
    else:
        a, b = x[..., :P], x[..., P:2 * P]
        r = torch.cat((a * c - b * sn, b * c + a * sn), -1)
    return torch.cat((r, x[..., 2 * P:]), -1).to(s["x"].dtype)


def _plain_append(s):
    kc, ks, vc, vs = s["arrays"]
    T, H, D = s["k"].shape
    page, slots = s["page"], s["slots"]
    pg, tok = slots // page, slots % page
    out = []
    for x, codes, scales, value in ((s["k"], kc, ks, False), (s["v"], vc, vs, True)):
        c, sc = _quant_mxfp4(x.float()) if s["fmt"] == "mxfp4" else _quant_hif4(x.float())
        c = _pack(c)
        sc = sc.to(torch.uint8) if s["fmt"] == "mxfp4" else sc.contiguous().view(torch.uint8)
        scales.view(-1, H, page, sc.shape[-1])[pg, :, tok] = sc
        if value:
            at = codes.view(-1, H, page // 16, 2, 8, 4, 2, D // 16)
            at[pg, :, tok // 16, tok // 8 % 2, :, tok // 2 % 4, tok % 2] = c.view(T, H, 8, D // 16)
            c = at[pg, :, tok // 16, tok // 8 % 2, :, tok // 2 % 4, tok % 2].reshape(T, H, D // 2)
        else:
            at = codes.view(-1, H, page, 4, D // 32, 4)
            at[pg, :, tok] = c.view(T, H, D // 32, 4, 4).transpose(2, 3)
            c = at[pg, :, tok].transpose(2, 3).reshape(T, H, D // 2)
        sc = scales.view(-1, H, page, sc.shape[-1])[pg, :, tok]
        v = _values_mxfp4(_unpack(c), sc.int()) if s["fmt"] == "mxfp4" else _values_hif4(_unpack(c), sc.contiguous().view(torch.int32))
        out.append(v.bfloat16())
    return {"k": out[0], "v": out[1]}


def _plain_attn(s):
    T, Hq, D = s["q"].shape
    kc, ks, vc, vs = s["arrays"]
    page, R, H = s["page"], s["table"].shape[0], kc.shape[1]
    G, n = Hq // H, s["most"]
    at = s["table"].long().clamp_min(0)
    get = lambda c, sc, value: _load(c[at], sc[at], page, D, s["fmt"], value).transpose(1, 2).flatten(2, 3)  # noqa: E731  [R, H, keys, D]
    start = s["start"].long() if s["start"] is not None else torch.arange(R + 1, device=at.device)
    new = start[1:] - start[:-1]
    i = torch.arange(n, device=at.device)
    row = (start[:-1, None] + i).clamp_max(T - 1)  # [R, n]
    q = s["q"][row].float().unflatten(2, (H, G)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [R, H, G n, D]
    w = torch.matmul(q, get(kc, ks, False).transpose(2, 3)).mul_(s["scale"])
    j = torch.arange(w.shape[-1], device=at.device)
    p = s["lens"].long()[:, None] - new[:, None] + i  # a query's position
    see = (j <= p[..., None]) & (j < s["lens"][:, None, None])
    if s["window"]:
        see &= j > p[..., None] - s["window"]
    w = w.unflatten(2, (G, n)).masked_fill_(~see[:, None, None], -math.inf).flatten(2, 3)
    m = w.amax(-1, keepdim=True)
    w = (w - m.clamp_min(-1e30)).exp_()
    l = w.sum(-1, keepdim=True)
    o = torch.matmul(w, get(vc, vs, True)) / torch.where(l > 0, l, 1)
    lse = torch.where(l > 0, m + l.log(), -math.inf)
    back = lambda t: t.unflatten(2, (G, n)).permute(0, 3, 1, 2, 4)[i < new[:, None]].flatten(1, 2)  # noqa: E731
    return {"o": back(o).to(torch.bfloat16), "lse": back(lse)[..., 0]}


def _plain_matvec(s):
    codes, sc = s["codes"], s["sc"]
    N, K = codes.shape[0], codes.shape[1] * 2
    n128 = -(-N // 128) * 128
    if s["fmt"] == "mxfp4":
        if s["scales"] == "mma":
            sc = sc.view(n128 // 128, K // 128, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(n128, K // 32)
        w = _values_mxfp4(_unpack(codes), sc.view(-1, K // 32)[:N].int())
    else:
        sc = sc.view(torch.int32)
        sc = sc.view(K // 64, n128)[:, :N].t() if s["scales"] == "mma" else sc.view(N, K // 64)
        w = _values_hif4(_unpack(codes), sc)
    return torch.matmul(s["x"].float(), w.t()).to(s["y"].dtype)


# ---------------------------------------------------------------- exact

def _exact_scale(fmt, raw):
    """float64 scale of each group of 4 elements [..., n / 4], from the stored bytes [..., bytes of a row]."""
    b = raw.long()
    if fmt == "mxfp4":
        return torch.pow(torch.full((), 2.0, dtype=torch.float64, device=b.device), (b - 127).double()).repeat_interleave(8, -1)
    w = b.reshape(*b.shape[:-1], -1, 4)
    macro = torch.pow(torch.full((), 2.0, dtype=torch.float64, device=b.device), (w[..., 0] // 4 - 48).double()) * (1 + (w[..., 0] % 4).double() / 4)
    out = []
    for sub in range(16):
        e = (w[..., 1] // 2 ** (sub // 2)) % 2 + (w[..., 2 + sub // 8] // 2 ** (sub % 8)) % 2
        out.append(macro * 0.25 * (2.0 ** e.double()))
    return torch.stack(out, -1).flatten(-2)


def _exact_code(fmt, code):
    k = code % 8
    if fmt == "mxfp4":
        mant, ex = (k % 2).double(), (k // 2)
        v = torch.where(ex > 0, (1 + mant / 2) * 2.0 ** (ex - 1).double(), mant / 2)
    else:
        v = k.double()
    return torch.where(code >= 8, -v, v)


def _exact_quant(fmt, x):
    """float64 [..., n] -> the float64 values that the format holds for it."""
    if fmt == "mxfp4":
        b = x.reshape(*x.shape[:-1], -1, 32)
        a = b.abs().amax(-1, keepdim=True)
        e = (torch.frexp(a)[1] - 1 - 2).clamp(-127, 127).double()
        y = b / 2.0 ** e
        grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
        up = torch.searchsorted(grid, y.abs().contiguous()).clamp(0, 7)
        dn = (up - 1).clamp_min(0)
        lo, hi = y.abs() - grid[dn], grid[up] - y.abs()
        k = torch.where(lo < hi, dn, torch.where(lo > hi, up, torch.where(dn % 2 == 0, dn, up)))
        return (torch.sign(b) * grid[k] * 2.0 ** e).reshape(x.shape)
    b = x.reshape(*x.shape[:-1], -1, 16, 4)
    a = b.abs().amax((-2, -1))
    byte = torch.arange(256, device=x.device)
    table = 2.0 ** (byte // 4 - 48).double() * (1 + (byte % 4).double() / 4)
    s = table[torch.searchsorted(7 * table, a.contiguous()).clamp_max(255)][..., None]
    sub = b.abs().amax(-1)
    t = torch.where(sub <= 1.75 * s, 0, torch.where(sub <= 3.5 * s, 1, 2)).reshape(*sub.shape[:-1], 8, 2)
    t = torch.where((t.amax(-1, keepdim=True) == 2) & (t < 1), 1, t).reshape(sub.shape)
    step = (0.25 * s * 2.0 ** t.double())[..., None]
    k = (b.abs() / step).clamp_max(7.0).round()
    return (torch.sign(b) * k * step).reshape(x.shape)


def _exact_cache(s, D, pages, value):
    """float64 [tokens, H, D] of a request's pages, each element found by its documented place."""
    codes, raw = (s["arrays"][2], s["arrays"][3]) if value else (s["arrays"][0], s["arrays"][1])
    page = s["page"]
    tok, d = torch.arange(page, device=codes.device)[:, None], torch.arange(D, device=codes.device)[None]
    if value:
        g, rest = d // (D // 8), d % (D // 8)
        byte = ((tok // 16 * 2 + tok % 16 // 8) * 8 + g) * (D // 2) + (tok % 8 // 2) * (D // 8) + (tok % 2) * (D // 16) + rest // 2
    else:
        byte = tok * (D // 2) + ((d % 32 // 8) * (D // 32) + d // 32) * 4 + d % 8 // 2
    c = codes[pages][:, :, byte.flatten()].long().reshape(len(pages), codes.shape[1], page, D)
    c = torch.where(d % 2 == 0, c % 16, c // 16)
    sc = _exact_scale(s["fmt"], raw[pages].reshape(len(pages), codes.shape[1], page, -1))
    v = _exact_code(s["fmt"], c) * sc.repeat_interleave(4, -1)
    return v.permute(0, 2, 1, 3).reshape(-1, codes.shape[1], D)


def exact(case, seed):
    op = case["op"]
    if op == "slots":
        return None  # whole numbers alone
    s = prepare(case, seed)
    if op == "rope":
        x, P = s["x"].double(), s["freq"].numel()
        th = (s["pos"].double()[s["axis"].long()] * s["freq"].double()[:, None]).t()
        z = torch.polar(torch.ones_like(th), -th if s["inverse"] else th)[:, None]
        if s["pair"] == 1:
            y = torch.view_as_real(torch.view_as_complex(x[..., :2 * P].reshape(*x.shape[:2], P, 2).contiguous()) * z).flatten(-2)
        else:
            w = torch.complex(x[..., :P], x[..., P:2 * P]) * z
            y = torch.cat((w.real, w.imag), -1)
        return torch.cat((y, x[..., 2 * P:]), -1)
    if op == "append":
        return {"k": _exact_quant(case["fmt"], s["k"].double()), "v": _exact_quant(case["fmt"], s["v"].double())}
    if op == "attn":
        lens, new = _lengths(case, seed)
        T, Hq, D = s["q"].shape
        G = Hq // case["kv"]
        o = torch.zeros(T, Hq, D, dtype=torch.float64, device=DEV)
        lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=DEV)
        t0 = 0
        for r, (L, n) in enumerate(zip(lens, new)):
            if L:
                pages = s["table"][r, :-(-L // case["page"])].long()
                k, v = (_exact_cache(s, D, pages, value)[:L] for value in (False, True))
                pos = L - n + torch.arange(n, device=DEV)[:, None]
                key = torch.arange(L, device=DEV)[None]
                hide = key > pos
                if case["window"]:
                    hide |= key <= pos - case["window"]
                for h in range(case["kv"]):
                    q = s["q"][t0:t0 + n, h * G:(h + 1) * G].double()
                    w = (torch.einsum("tgd,kd->tgk", q, k[:, h]) * D ** -0.5).masked_fill(hide[:, None], -math.inf)
                    z = torch.logsumexp(w, -1)
                    lse[t0:t0 + n, h * G:(h + 1) * G] = z
                    w = torch.exp(w - torch.where(z > -math.inf, z, 0.0)[..., None])
                    o[t0:t0 + n, h * G:(h + 1) * G] = torch.einsum("tgk,kd->tgd", w, v[:, h])
            t0 += n
        return {"o": o, "lse": lse}
    K, N = case["k"], case["n"]
    raw, n128 = s["sc"], -(-N // 128) * 128
    y = torch.empty(case["rows"], N, dtype=torch.float64, device=DEV)
    x = s["x"].double()
    for r0 in range(0, N, 4096):
        n = torch.arange(r0, min(N, r0 + 4096), device=DEV)[:, None]
        if case["fmt"] == "mxfp4":
            b = torch.arange(K // 32, device=DEV)[None]
            at = (n // 128 * (K // 128) + b // 4) * 512 + n % 32 * 16 + n // 32 % 4 * 4 + b % 4 if case["scales"] == "mma" else n * (K // 32) + b
        else:
            b = torch.arange(K // 16, device=DEV)[None]
            at = ((b // 4) * n128 + n) * 4 + b % 4 if case["scales"] == "mma" else n * (K // 16) + b
        c = s["codes"][r0:r0 + 4096].long()
        c = torch.stack((c % 16, c // 16), -1).flatten(-2)
        y[:, r0:r0 + 4096] = x @ (_exact_code(case["fmt"], c) * _exact_scale(case["fmt"], raw[at]).repeat_interleave(4, -1)).t()
    return y


# ---------------------------------------------------------------- work

def work(case):
    """Bytes and operations that a pass cannot do without (lengths as one seed gives them)."""
    op = case["op"]
    if op == "slots":
        R, tokens = case["requests"], sum(max(0, a) for a in _step(case, 0)[1])
        return {"bytes": 16 * R + 12 * tokens + 8 * (tokens // case["page"]), "flops": 0}
    if op == "rope":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": n * 2 * (2 if case["dtype"] == "bf16" else 4) + 4 * case["tokens"] * case["axes"], "flops": 3 * n}
    each = 0.5 + (1 / 32 if case["fmt"] == "mxfp4" else 1 / 16)
    if op == "append":
        n = 2 * case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": n * (2 + each) + n * (each + 2) + 16 * case["tokens"], "flops": 2 * n}
    if op == "attn":
        lens, new = _lengths(case, 0)
        keys = pairs = 0
        for L, n in zip(lens, new):
            w = case["window"] or L + 1
            first = max(0, L - n + 1 - w)
            keys += L - min(first, L)
            for p in range(max(0, L - n), L):
                pairs += min(p + 1, w)
        T = sum(new)
        return {"bytes": keys * case["kv"] * 2 * case["dim"] * each + T * case["heads"] * (4 * case["dim"] + 4),
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    M, K, N = case["rows"], case["k"], case["n"]
    return {"bytes": N * K * each + 2 * M * K + M * N * (2 if case["out"] == "bf16" else 4), "flops": 2 * M * N * K}
