"""Cases for the operators around a mixture-of-experts block, and the plain
forms their results are held against.

  norm      layer and RMS norm of rows or heads, and their gradients
  route     the router: top_k of the experts' logits and their weights, and its gradient
  dispatch  pairs (token, expert) sorted by expert, and the tokens' rows brought to their groups
  combine   the experts' rows brought back, weighted and summed, and its gradient
  quantize  the dispatch that quantizes each token once into the 4-bit groups of the grouped product

``run`` computes a case in elementary torch operations in 32 bits, or through
the library's entry points where ``own`` is set.
"""
import math
import random

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
EPS = 1e-6


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # the affine layer norm of a Wan2.2-14B DiT block over a whole clip, statistics kept for the backward pass
        {"name": "norm video", "op": "norm", "tokens": 32760, "heads": 1, "row": 1, "dim": 5120, "kind": "layer", "affine": "both",
         "stats": True, "back": False, "dtype": "bf16"},
        # RMS norm of the query and key heads inside the packed projection of a Qwen3-VL layer
        {"name": "norm heads", "op": "norm", "tokens": 4096, "heads": 40, "row": 48, "dim": 128, "kind": "rms", "affine": "weight",
         "stats": False, "back": False, "dtype": "bf16"},
        # the backward pass of the first: gradients of x, of the weight and of the bias
        {"name": "norm gradient", "op": "norm", "tokens": 32760, "heads": 1, "row": 1, "dim": 5120, "kind": "layer", "affine": "both",
         "stats": True, "back": True, "dtype": "bf16"},
        # a short batch in fp32 whose rows are of no convenient length
        {"name": "norm gradient odd", "op": "norm", "tokens": 1531, "heads": 1, "row": 1, "dim": 1023, "kind": "rms", "affine": "weight",
         "stats": True, "back": True, "dtype": "f32"},
        # one token of each request of a decoding step through the router of Qwen3-VL-30B-A3B: latency
        {"name": "route decode", "op": "route", "tokens": 61, "experts": 128, "top_k": 8, "normalize": True, "masked": 0, "back": False,
         "dtype": "bf16"},
        # the router's gradient over a training batch, some experts switched off for some tokens
        {"name": "route gradient", "op": "route", "tokens": 32768, "experts": 128, "top_k": 8, "normalize": False, "masked": 5, "back": True,
         "dtype": "f32"},
        # the tokens of a decoding step brought to their experts, two of the step's places empty
        {"name": "dispatch decode", "op": "dispatch", "tokens": 32, "spare": 2, "dim": 2048, "experts": 128, "top_k": 8, "align": 1, "dtype": "bf16"},
        # a prompt's tokens stacked for the grouped product: groups on 128-row boundaries, zeros between
        {"name": "dispatch prompt", "op": "dispatch", "tokens": 4096, "spare": 0, "dim": 2048, "experts": 128, "top_k": 8, "align": 128,
         "dtype": "bf16"},
        # the experts' rows of the same prompt brought back
        {"name": "combine prompt", "op": "combine", "tokens": 4096, "spare": 0, "dim": 2048, "experts": 128, "top_k": 8, "align": 128,
         "back": False, "dtype": "bf16"},
        # gradients of the experts' rows and of the router's weights, ragged sizes in fp32
        {"name": "combine gradient", "op": "combine", "tokens": 3001, "spare": 13, "dim": 1000, "experts": 60, "top_k": 6, "align": 16,
         "back": True, "dtype": "f32"},
        # a small batch quantized into its experts' groups, rows of no token left alone
        {"name": "quantize decode", "op": "quantize", "tokens": 16, "spare": 0, "dim": 2048, "experts": 128, "top_k": 8, "align": 128,
         "zeros": False, "residual": True},
        # a prompt with its residual pathway, every row written
        {"name": "quantize prompt", "op": "quantize", "tokens": 4096, "spare": 96, "dim": 2048, "experts": 128, "top_k": 8, "align": 128,
         "zeros": True, "residual": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm", "route", "route", "dispatch", "combine", "combine", "quantize"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        heads = rng.choice([1, 1, 1, rng.randint(2, 40)])
        dim = rng.choice([64, 80, 128, 128]) if heads > 1 else rng.choice([_log(rng, 16, 13824), 8 * _log(rng, 2, 1728), 8 * _log(rng, 2, 1728)])
        tokens = _log(rng, 1, min(32768, 2 ** 26 // (heads * dim)))
        return {"op": op, "tokens": tokens, "heads": heads, "row": heads + (rng.choice([0, 8]) if heads > 1 else 0), "dim": dim,
                "kind": rng.choice(["layer", "rms"]), "affine": rng.choice(["both", "weight", "none"]), "stats": rng.random() < 0.5,
                "back": rng.random() < 0.5, "dtype": dtype}
    if op == "route":
        experts = rng.choice([8, 16, 60, 64, 128, 160, 256])
        top_k = rng.choice([1, 2, 4, 6, 8])
        return {"op": op, "tokens": _log(rng, 1, 32768), "experts": experts, "top_k": top_k,
                "normalize": top_k > 1 and rng.random() < 0.5, "masked": rng.choice([0, 0, 5]), "back": rng.random() < 0.5, "dtype": dtype}
    experts = rng.choice([8, 16, 60, 64, 128])
    top_k = rng.choice([1, 2, 4, 6, 8])
    tokens = _log(rng, 1, 4096)
    c = {"op": op, "tokens": tokens, "spare": rng.choice([0, 0, tokens // 16]), "dim": rng.choice([_log(rng, 16, 2048), 8 * _log(rng, 8, 256)]),
         "experts": experts, "top_k": top_k, "align": rng.choice([1, 16, 128, 128])}
    if op == "dispatch":
        return {**c, "dtype": dtype}
    if op == "combine":
        return {**c, "back": rng.random() < 0.5, "dtype": dtype}
    return {**c, "dim": 128 * rng.randint(1, 16), "align": 128, "zeros": rng.random() < 0.5, "residual": rng.random() < 0.7}


# ---------------------------------------------------------------- prepare

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _activations(g, shape):
    """fp32 values as a layer gives them (exact in bf16): some channels stand out, and their mean is not zero."""
    x = torch.randn(shape, generator=g, device=DEV)
    c = 1 + 15 * (torch.rand(shape[-1], generator=g, device=DEV) < 0.02).float()
    return (x * c + 0.3 * torch.randn(shape[-1], generator=g, device=DEV)).bfloat16().float()


def _rows(case):
    """Rows that hold a case's groups whatever the router says."""
    pairs = case["tokens"] * case["top_k"]
    return -(-(pairs + min(pairs, case["experts"]) * (case["align"] - 1)) // case["align"]) * case["align"]


def _ids(g, case):
    """The experts of each token, int32 [tokens, top_k]: some experts are liked better; the last `spare` tokens have none."""
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    like = torch.randn(T, E, generator=g, device=DEV) + 0.5 * torch.randn(E, generator=g, device=DEV)
    ids = like.topk(k, -1).indices.int()
    ids[T - case["spare"]:] = -1
    return ids


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    if op == "norm":
        T, H, R, D, dt = case["tokens"], case["heads"], case["row"], case["dim"], _type(case)
        s = {"op": op, "kind": case["kind"], "back": case["back"], "x": _activations(g, (T, R, D)).to(dt)[:, :H]}
        s["weight"] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) if case["affine"] != "none" else None
        s["bias"] = (0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) if case["affine"] == "both" else None
        new = lambda: torch.empty(T, H, D, dtype=dt, device=DEV)  # noqa: E731
        if not case["back"]:
            s["y"] = new()
            s["rstd"] = torch.zeros(T, H, device=DEV) if case["stats"] else None
            s["mean"] = torch.zeros(T, H, device=DEV) if case["stats"] and case["kind"] == "layer" else None
            return s
        x = s["x"].double()
        mean = x.mean(-1) if case["kind"] == "layer" else torch.zeros(T, H, dtype=torch.float64, device=DEV)
        s["rstd"] = ((x - mean[..., None]).square().mean(-1) + EPS).rsqrt().float().contiguous()
        s["mean"] = mean.float().contiguous() if case["kind"] == "layer" else None
        s["dy"], s["dx"] = torch.randn(T, H, D, generator=g, device=DEV).to(dt), new()
        s["dw"] = torch.empty(D, dtype=torch.float32, device=DEV) if case["affine"] != "none" else None
        s["db"] = torch.empty(D, dtype=torch.float32, device=DEV) if case["affine"] == "both" else None
        if own:
            from paper_2608_26581_gb300 import rfq
            s["ws"] = rfq.norm_workspace(D)
        return s
    if op == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        logits = (2 * torch.randn(T, E, generator=g, device=DEV) + 0.5 * torch.randn(E, generator=g, device=DEV)).to(_type(case))
        if case["masked"]:  # one expert in so many is off for a token, and now and then all are
            off = torch.rand(T, E, generator=g, device=DEV) * case["masked"] < 1
            off |= (torch.rand(T, 1, generator=g, device=DEV) < 0.01)
            logits = logits.masked_fill(off, -math.inf)
        s = {"op": op, "back": case["back"], "normalize": case["normalize"], "logits": logits,
             "ids": torch.empty(T, k, dtype=torch.int32, device=DEV), "weights": torch.empty(T, k, device=DEV)}
        if case["back"]:
            top, at = logits.float().sort(dim=-1, descending=True, stable=True)
            s["ids"].copy_(torch.where(top[:, :k] > -math.inf, at[:, :k], -1))
            s["dweights"], s["dlogits"] = torch.randn(T, k, generator=g, device=DEV), torch.empty_like(logits)
        return s
    T, D, E, k, n = case["tokens"], case["dim"], case["experts"], case["top_k"], _rows(case)
    s = {"op": op, "experts": E, "align": case["align"], "ids": _ids(g, case)}
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    s["off"], s["row_of"], s["pair_of"], s["ws"] = i32(E + 1), i32(T, k), i32(n), i32(64)
    if op == "dispatch":
        s["x"], s["out"] = _activations(g, (T, D)).to(_type(case)), torch.zeros(n, D, dtype=_type(case), device=DEV)
        return s
    _, s["row_of"], s["pair_of"] = _sorted(s["ids"], E, case["align"], n)
    if op == "combine":
        dt = _type(case)
        s |= {"back": case["back"], "y": _activations(g, (n, D)).to(dt), "weights": torch.rand(T, k, generator=g, device=DEV) / k}
        if case["back"]:
            s |= {"dout": torch.randn(T, D, generator=g, device=DEV).to(dt), "dy": torch.zeros(n, D, dtype=dt, device=DEV),
                  "dweights": torch.zeros(T, k, device=DEV)}
        else:
            s["out"] = torch.empty(T, D, dtype=dt, device=DEV)
        return s
    s |= {"x": _activations(g, (T, D)).bfloat16(), "zeros": case["zeros"], "residual": case["residual"]}
    s["main"] = torch.zeros(n, D, dtype=torch.bfloat16, device=DEV)
    s["res"] = torch.zeros(n, D, dtype=torch.bfloat16, device=DEV) if case["residual"] else None
    if own:
        from paper_2608_26581_gb300 import rfq
        for name in ("xq", "xr") if case["residual"] else ("xq",):
            s[name] = rfq.empty_qtensor(rfq.RFQ_FMT_MXFP4, rfq.RFQ_SCALE_MMA, n, D, device=DEV)
            s[name].codes.zero_()
            s[name].scales.zero_()
    return s


# ---------------------------------------------------------------- run

def run(s):
    if own:
        return _own(s)
    return {"norm": _plain_norm, "route": _plain_route, "dispatch": _plain_dispatch, "combine": _plain_combine,
            "quantize": _plain_quantize}[s["op"]](s)


def _own(s):
    from paper_2608_26581_gb300 import rfq
    if s["op"] == "norm":
        kind = rfq.RFQ_NORM_LAYER if s["kind"] == "layer" else rfq.RFQ_NORM_RMS
        if s["back"]:
            rfq.rfq_norm_grad(s["dy"], s["x"], s["rstd"], s["dx"], mean=s["mean"], weight=s["weight"], dweight=s["dw"], dbias=s["db"],
                              workspace=s["ws"], kind=kind)
            return {n: s[n] for n in ("dx", "dw", "db") if s[n] is not None}
        rfq.rfq_norm(s["x"], s["y"], weight=s["weight"], bias=s["bias"], kind=kind, eps=EPS, mean=s["mean"], rstd=s["rstd"])
        return {n: s[n] for n in ("y", "mean", "rstd") if s[n] is not None}
    if s["op"] == "route":
        if s["back"]:
            rfq.rfq_route_grad(s["logits"], s["ids"], s["dweights"], s["dlogits"], normalize=s["normalize"])
            return {"dlogits": s["dlogits"]}
        rfq.rfq_route(s["logits"], s["ids"], s["weights"], normalize=s["normalize"])
        return {"ids": s["ids"], "weights": s["weights"]}
    if s["op"] == "dispatch":
        rfq.rfq_moe_sort(s["ids"], s["off"], s["row_of"], s["pair_of"], s["ws"], align=s["align"])
        rfq.rfq_moe_gather(s["x"], s["row_of"], s["out"], pair_of=s["pair_of"])
        return {n: s[n] for n in ("off", "row_of", "pair_of", "out")}
    if s["op"] == "combine":
        if s["back"]:
            rfq.rfq_moe_combine_grad(s["dout"], s["y"], s["row_of"], s["weights"], s["dy"], s["dweights"], pair_of=s["pair_of"])
            return {"dy": s["dy"], "dweights": s["dweights"]}
        rfq.rfq_moe_combine(s["y"], s["row_of"], s["out"], weights=s["weights"])
        return {"out": s["out"]}
    rfq.rfq_moe_quantize(s["x"], s["row_of"], s["xq"], s.get("xr"), pair_of=s["pair_of"] if s["zeros"] else None)
    rfq.rfq_dequant(s["xq"], s["main"])
    if not s["residual"]:
        return {"main": s["main"]}
    rfq.rfq_dequant(s["xr"], s["res"])
    return {"main": s["main"], "residual": s["res"]}


def _plain_norm(s):
    x = s["x"].float()
    w = s["weight"].float() if s["weight"] is not None else torch.ones(x.shape[-1], device=x.device)
    if s["back"]:
        dy = s["dy"].float()
        xh = (x if s["mean"] is None else x - s["mean"][..., None]) * s["rstd"][..., None]
        g = dy * w
        dx = g - xh * (g * xh).mean(-1, keepdim=True)
        if s["kind"] == "layer":
            dx = dx - g.mean(-1, keepdim=True)
        out = {"dx": (dx * s["rstd"][..., None]).to(s["x"].dtype)}
        if s["dw"] is not None:
            out["dw"] = (dy * xh).sum((0, 1))
        if s["db"] is not None:
            out["db"] = dy.sum((0, 1))
        return out
    mean = x.mean(-1) if s["kind"] == "layer" else torch.zeros(x.shape[:-1], device=x.device)
    d = x - mean[..., None]
    rstd = 1 / (d.square().mean(-1) + EPS).sqrt()
    y = d * rstd[..., None] * w
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    return {n: out[n] for n in out if s[n] is not None}


def _plain_route(s):
    logits, k = s["logits"].float(), s["ids"].shape[1]
    if not s["back"]:
        top, at = logits.sort(dim=-1, descending=True, stable=True)
        most, top, at = top[:, :1].clamp_min(-1e30), top[:, :k], at[:, :k]
        e = (top - most).exp()
        whole = e.sum(-1, keepdim=True) if s["normalize"] else (logits - most).exp().sum(-1, keepdim=True)
        return {"ids": torch.where(top > -math.inf, at, -1).int(), "weights": e / torch.where(whole > 0, whole, 1)}
    ids = s["ids"].long()
    there = ids >= 0
    taken = torch.zeros(logits.shape[0], logits.shape[1] + 1, device=logits.device)
    d = taken.scatter(1, torch.where(there, ids, logits.shape[1]), s["dweights"])[:, :-1]
    taken = taken.scatter(1, torch.where(there, ids, logits.shape[1]), 1.0)[:, :-1]
    e = (logits - logits.amax(-1, keepdim=True).clamp_min(-1e30)).exp()
    if s["normalize"]:
        e = e * taken
    whole = e.sum(-1, keepdim=True)
    p = e / torch.where(whole > 0, whole, 1)
    d = d * taken
    return {"dlogits": (p * (d - (p * d).sum(-1, keepdim=True))).to(s["logits"].dtype)}


def _sorted(ids, experts, align, rows):
    """Group offsets, the row of each pair, the pair of each row."""
    flat = ids.flatten().long()
    key, order = torch.where((flat >= 0) & (flat < experts), flat, experts).sort(stable=True)
    first = torch.searchsorted(key, torch.arange(experts + 1, device=ids.device))
    end = ((first[1:] - first[:-1] + align - 1) // align * align).cumsum(0)
    off = torch.cat((torch.zeros(1, dtype=torch.int64, device=ids.device), end))
    at = torch.arange(flat.numel(), device=ids.device) + (off - first)[key]
    there = key < experts
    row = torch.empty_like(flat)
    row[order] = torch.where(there, at, -1)
    pair = torch.full((rows + 1,), -1, dtype=torch.int32, device=ids.device)
    pair[torch.where(there, at, rows)] = order.int()
    return off.int(), row.int().view(ids.shape), pair[:-1].contiguous()


def _scattered(v, row_of, rows):
    """Each token's row of v at the rows of its pairs, zeros elsewhere."""
    out = torch.zeros(rows + 1, v.shape[-1], dtype=v.dtype, device=v.device)
    at = torch.where(row_of >= 0, row_of, rows).long()
    out[at.flatten()] = v.repeat_interleave(row_of.shape[1], 0)
    return out[:-1]


def _plain_dispatch(s):
    off, row_of, pair_of = _sorted(s["ids"], s["experts"], s["align"], s["pair_of"].numel())
    return {"off": off, "row_of": row_of, "pair_of": pair_of, "out": _scattered(s["x"], row_of, pair_of.numel())}


def _plain_combine(s):
    there = s["row_of"] >= 0
    y = s["y"].float()[s["row_of"].long().clamp_min(0)]  # [T, k, D]
    w = s["weights"] * there
    if not s["back"]:
        return {"out": (y * w[..., None]).sum(1).to(s["y"].dtype)}
    dout = s["dout"].float()[:, None]
    dy = torch.zeros(s["y"].shape[0] + 1, s["y"].shape[1], dtype=s["y"].dtype, device=y.device)
    dy[torch.where(there, s["row_of"], s["y"].shape[0]).long()] = (w[..., None] * dout).to(dy.dtype)
    return {"dy": dy[:-1], "dweights": (y * dout).sum(-1) * there}


E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values_mxfp4(x):
    """fp32 [..., n] (n % 32 == 0) -> the fp32 values that MXFP4 holds for it."""
    b = x.unflatten(-1, (-1, 32))
    e = ((b.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp_min(0)
    s = torch.where(e > 0, e << 23, torch.full_like(e, 0x400000)).view(torch.float32).unsqueeze(-1)
    y = b.abs() / s
    # the grid of E2M1: steps of 1/2 below 2, of 1 below 4, of 2 above; ties to even
    k = torch.where(y < 2, (y * 2).round(), torch.where(y < 4, y.round() + 2, (y / 2).round() + 4)).clamp_max(7).long()
    return (torch.tensor(E2M1, device=x.device)[k] * s).copysign(b).flatten(-2)


def _plain_quantize(s):
    x = s["x"].float()
    v = _values_mxfp4(x)
    n = s["pair_of"].numel()
    out = {"main": _scattered(v.bfloat16(), s["row_of"], n)}
    if s["residual"]:
        out["residual"] = _scattered(_values_mxfp4(x - v).bfloat16(), s["row_of"], n)
    return out


# ---------------------------------------------------------------- exact

def _exact_mxfp4(x):
    """float64 [..., n] -> the float64 values that MXFP4 holds for it."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    e = (torch.frexp(b.abs().amax(-1, keepdim=True))[1] - 3).clamp(-127, 127).long()
    s = (e + 1023 << 52).view(torch.float64)  # (a power taken on the GPU may be a bit off)
    y = b.abs() / s
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    up = torch.searchsorted(grid, y.contiguous()).clamp(0, 7)
    dn = (up - 1).clamp_min(0)
    lo, hi = y - grid[dn], grid[up] - y
    k = torch.where(lo < hi, dn, torch.where(lo > hi, up, torch.where(dn % 2 == 0, dn, up)))
    return (torch.sign(b) * grid[k] * s).reshape(x.shape)


def _exact_norm(case, s):
    x = s["x"].double()
    D = x.shape[-1]
    w = s["weight"].double() if s["weight"] is not None else None
    if case["back"]:
        dy, r = s["dy"].double(), s["rstd"].double()[..., None]
        xh = x * r if s["mean"] is None else (x - s["mean"].double()[..., None]) * r
        out = {"dw": torch.einsum("thd,thd->d", dy, xh) if s["dw"] is not None else None,
               "db": torch.einsum("thd->d", dy) if s["db"] is not None else None}
        g = dy if w is None else dy * w
        along = torch.einsum("thd,thd->th", g, xh)[..., None]
        even = torch.einsum("thd->th", g)[..., None] if case["kind"] == "layer" else 0.0
        return {"dx": r / D * (D * g - even - xh * along), **out}
    if case["kind"] == "layer":
        var, mean = torch.var_mean(x, -1, unbiased=False)
    else:
        mean, var = torch.zeros(x.shape[:-1], dtype=torch.float64, device=DEV), torch.einsum("thd,thd->th", x, x) / D
    rstd = (var + EPS) ** -0.5
    y = (x - mean[..., None]) * rstd[..., None]
    y = y if w is None else y * w
    y = y if s["bias"] is None else y + s["bias"].double()
    out = {"y": y, "mean": mean, "rstd": rstd}
    return {n: out[n] for n in out if s[n] is not None}


def _exact_route(case, s):
    logits, k = s["logits"].double(), case["top_k"]
    if case["back"]:  # by the formula's own Jacobian, over the taken ones
        there = s["ids"] >= 0
        at = s["ids"].long().clamp_min(0)
        l = torch.gather(logits, 1, at).masked_fill(~there, -math.inf)
        z = torch.logsumexp(l if case["normalize"] else logits, -1, keepdim=True)
        w = torch.where(there, torch.exp(l - torch.where(z > -math.inf, z, 0.0)), 0.0)
        dot = (w * s["dweights"].double()).sum(-1, keepdim=True)
        if case["normalize"]:
            d = torch.zeros_like(logits)
        else:
            d = -torch.exp(logits - torch.where(z > -math.inf, z, 0.0)) * dot
        at = torch.where(there, at, 0)
        return {"dlogits": d.scatter_add(1, at, torch.where(there, w * (s["dweights"].double() - (dot if case["normalize"] else 0.0)), 0.0))}
    l = torch.topk(logits, k, -1).values
    z = torch.logsumexp(l if case["normalize"] else logits, -1, keepdim=True)
    return {"ids": None, "weights": torch.exp(l - torch.where(z > -math.inf, z, 0.0))}


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if op == "norm":
        return _exact_norm(case, s)
    if op == "route":
        return _exact_route(case, s)
    T, k, n = case["tokens"], case["top_k"], s["pair_of"].numel()
    if op == "dispatch":  # each pair counts those before it
        flat = s["ids"].flatten().long()
        mine = flat[:, None] == torch.arange(case["experts"], device=DEV)
        nth = torch.cumsum(mine, 0)
        whole = -(-nth[-1] // case["align"]) * case["align"]
        at = (nth - 1 + torch.cumsum(whole, 0) - whole)[mine]
        out = torch.zeros(n, case["dim"], dtype=torch.float64, device=DEV)
        out[at] = s["x"].double()[torch.nonzero(flat >= 0).flatten() // k]
        return {"off": None, "row_of": None, "pair_of": None, "out": out}
    pair = s["pair_of"].long()
    rows = torch.nonzero(pair >= 0).flatten()
    pair = pair[rows]
    if op == "combine":
        y, w = s["y"].double()[rows], s["weights"].double().flatten()[pair]
        if not case["back"]:
            return {"out": torch.zeros(T, case["dim"], dtype=torch.float64, device=DEV).index_add(0, pair // k, y * w[:, None])}
        dout = s["dout"].double()[pair // k]
        dy = torch.zeros(n, case["dim"], dtype=torch.float64, device=DEV)
        dy[rows] = dout * w[:, None]
        dw = torch.zeros(T * k, dtype=torch.float64, device=DEV)
        dw[pair] = torch.einsum("rd,rd->r", dout, y)
        return {"dy": dy, "dweights": dw.view(T, k)}
    x = s["x"].double()
    main = _exact_mxfp4(x)
    out = {}
    for name, v in (("main", main), ("residual", _exact_mxfp4(x - main) if case["residual"] else None)):
        if v is not None:
            out[name] = torch.zeros(n, case["dim"], dtype=torch.float64, device=DEV)
            out[name][rows] = v[pair // k]
    return out


# ---------------------------------------------------------------- work

def work(case):
    """Bytes and operations that a pass cannot do without."""
    op = case["op"]
    size = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if op == "norm":
        rows = case["tokens"] * case["heads"]
        n = rows * case["dim"]
        side = {"both": 2, "weight": 1, "none": 0}[case["affine"]] * case["dim"]
        if case["back"]:
            return {"bytes": 3 * n * size + 8 * rows + side * 4 + case["dim"] * size, "flops": 12 * n}
        return {"bytes": 2 * n * size + ((8 if case["kind"] == "layer" else 4) * rows if case["stats"] else 0) + side * size, "flops": 7 * n}
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    if op == "route":
        if case["back"]:
            return {"bytes": 2 * T * E * size + 8 * T * k, "flops": 6 * T * E}
        return {"bytes": T * E * size + 8 * T * k, "flops": (3 + k) * T * E}
    D, rows, pairs = case["dim"], _rows(case), (T - case["spare"]) * k
    if op == "dispatch":
        return {"bytes": T * k * 8 + E * 4 + rows * 4 + (T + rows) * D * size, "flops": 0}
    if op == "combine":
        if case["back"]:
            return {"bytes": (T + pairs + rows) * D * size + T * k * 12 + rows * 4, "flops": 3 * pairs * D}
        return {"bytes": (T + pairs) * D * size + T * k * 8, "flops": 2 * pairs * D}
    ways = 2 if case["residual"] else 1
    stored = rows if case["zeros"] else pairs
    return {"bytes": T * D * 2 + T * k * 4 + ways * D * ((stored + rows) * 17 / 32 + rows * 2), "flops": 4 * ways * T * D}
