"""Plain references of the entry points around a mixture-of-experts block, in
64 bits on the CPU, and bounds of what fp32 arithmetic may be off by.

u = 2^-24 is half a step of fp32.  No sum of the kernels chains more than CHAIN
additions (a lane's own, those over lanes, warps and blocks), so a sum is off
by at most CHAIN u times the sum of its terms' magnitudes, beside what its terms
are off by.  A result rounded to type t is off by finfo(t).eps / 2 of itself."""
import numpy as np
import torch

U = 2.0 ** -24
CHAIN = 128


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def norm(x, w, b, eps, rms):
    """float64 [..., dim] -> y, mean, rstd."""
    m = x.mean(-1) if not rms else torch.zeros_like(x[..., 0])
    d = x - m[..., None]
    r = (d.square().mean(-1) + eps) ** -0.5
    y = d * r[..., None]
    return (y if w is None else y * w) + (0 if b is None else b), m, r


def norm_bound(x, w, b, eps, rms, dtype):
    """How far y (of `dtype`), mean and rstd may be off.  The mean is off by
    CHAIN u mean|x| and its own two roundings; the variance by that of its terms
    (twice the mean's share, and CHAIN + 4 roundings), the root halves it."""
    y, m, r = norm(x, w, b, eps, rms)
    em = torch.zeros_like(m) if rms else (CHAIN + 2) * U * x.abs().mean(-1)
    h = (x - m[..., None]).abs() * r[..., None]
    # sum of 2 |d| em over n, against the variance + eps >= mean(d^2): h's mean times 2 em r
    er = r * (0.5 * (CHAIN + 8) * U + h.mean(-1) * em * r + (em * r) ** 2)
    wa = torch.ones_like(y) if w is None else w.abs().expand_as(y)
    ey = wa * (r * em)[..., None] + wa * h * ((er / r)[..., None] + 6 * U) + 2 * U * y.abs() + half_step(dtype) * y.abs()
    if b is not None:
        ey = ey + 2 * U * b.abs()
    return ey, em, er


def norm_grad(dy, x, m, r, w, rms):
    """float64 -> dx, dw, db (sums over all leading axes)."""
    h = (x if rms else x - m[..., None]) * r[..., None]
    g = dy if w is None else dy * w
    dx = g - h * (g * h).mean(-1, keepdim=True)
    if not rms:
        dx = dx - g.mean(-1, keepdim=True)
    lead = tuple(range(x.dim() - 1))
    return dx * r[..., None], (dy * h).sum(lead), dy.sum(lead)


def norm_grad_bound(dy, x, m, r, w, rms, dtype):
    """h is off by 3 u of itself and, by the difference, u (|x| + |m|) r; g by u; the
    means by their chains and their terms; four more roundings; then the type's."""
    d = x if rms else x - m[..., None]
    h, R = (d * r[..., None]).abs(), r[..., None]
    eh = 4 * U * h
    g = (dy if w is None else dy * w).abs()
    gh = (g * h).mean(-1, keepdim=True)
    mean_g = torch.zeros_like(gh) if rms else g.mean(-1, keepdim=True)
    e_gh = (CHAIN + 8) * U * gh
    dx = norm_grad(dy, x, m, r, w, rms)[0]
    ex = R * (2 * U * g + (CHAIN + 4) * U * mean_g + h * e_gh + (eh + 2 * U * h) * gh + 4 * U * (g + mean_g + h * gh)) + half_step(dtype) * dx.abs()
    lead = tuple(range(x.dim() - 1))
    return ex, (CHAIN + 8) * U * (dy.abs() * h).sum(lead), (CHAIN + 2) * U * dy.abs().sum(lead)


def route(logits, k, normalize):
    """float64 [T, E] -> ids int [T, k], weights: choice by choice."""
    T, E = logits.shape
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        row = logits[t].numpy()
        # (NaN counts as the largest; it and +inf make the weights NaN)
        order = sorted((e for e in range(E) if row[e] != -np.inf), key=lambda e: (not np.isnan(row[e]), -row[e], e))[:k]
        if order:
            with np.errstate(invalid="ignore"):
                e = np.exp(row - row[order[0]])
            z = e[order].sum() if normalize else e.sum()
            ids[t, :len(order)], w[t, :len(order)] = order, e[order] / z
    return torch.from_numpy(ids), torch.from_numpy(w)


def softmax_over(logits, ids, normalize):
    """p over all experts or the chosen ones, and the bound of its relative
    error: l - m is off by u |l - m|, the exponential by 2 steps more, their sum
    by its terms and its chain, the quotient by 2 u."""
    T, E = logits.shape
    taken = torch.zeros(T, E + 1, dtype=torch.bool)
    taken.scatter_(1, torch.where((ids >= 0) & (ids < E), ids, E).long(), True)
    l = logits.masked_fill(~taken[:, :-1], -np.inf) if normalize else logits
    m = l.amax(-1, keepdim=True).clamp_min(-1e300)
    e = torch.exp(l - m)
    z = e.sum(-1, keepdim=True)
    p = e / torch.where(z > 0, z, 1)
    far = torch.where(torch.isfinite(l), m - l, 0.0)
    rel = U * (far + (p * far).sum(-1, keepdim=True) + CHAIN + 12)
    return p, rel


def route_grad(logits, ids, dw, normalize):
    """float64 -> dlogits and the bound of what fp32 (before the last rounding) is off by."""
    T, E = logits.shape
    p, rel = softmax_over(logits, ids, normalize)
    d = torch.zeros(T, E + 1, dtype=torch.float64).scatter_add_(1, torch.where((ids >= 0) & (ids < E), ids, E).long(), dw)[:, :-1]
    s = (p * d).sum(-1, keepdim=True)
    es = (p * d.abs() * (rel + (CHAIN + 2) * U)).sum(-1, keepdim=True)
    return p * (d - s), p * (rel * (d - s).abs() + es + 3 * U * (d.abs() + s.abs())) + 2.0 ** -149


def sort(ids, experts, align, rows):
    """Pair by pair: group_off, row_of, pair_of, and whether all pairs found a row."""
    flat = ids.flatten().tolist()
    groups = [[p for p, e in enumerate(flat) if e == g] for g in range(experts)]
    most = rows // align * align
    off, row_of, pair_of, at = [0], np.full(len(flat), -1, np.int32), np.full(rows, -1, np.int32), 0
    for g in groups:
        for i, p in enumerate(g):
            if at + i < most:
                row_of[p], pair_of[at + i] = at + i, p
        at += -(-len(g) // align) * align
        off.append(min(at, most))
    return torch.tensor(off, dtype=torch.int32), torch.from_numpy(row_of).view(ids.shape), torch.from_numpy(pair_of), at <= most
