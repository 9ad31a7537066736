"""Plain references of the serving entry points, in 64 bits on the CPU:
a request-by-request slot allocator, the rotation of pairs, the cache's
documented layout, and softmax attention key by key."""
import numpy as np

FMT_MXFP4, FMT_HIF4 = 0, 1


def slot_map(cached, added, page, table, free, count, tokens):
    """One serving step, request by request; returns the new (table, free,
    count, lengths, token_start, slots, positions, bad)."""
    table, free = table.copy(), free.copy()
    R, width = table.shape
    pages = lambda n: -(-n // page)  # noqa: E731
    bad = False
    fits, after = [], []
    for c, a in zip(cached, added):
        n = max(c + a, 0)
        ok = c >= 0 and pages(c) <= width and pages(n) <= width
        bad |= not ok
        fits.append(ok)
        after.append(n)
    for r in range(R):
        if fits[r]:
            for j in range(pages(after[r]), pages(max(cached[r], 0))):
                if count < len(free):
                    free[count] = table[r, j]
                    count += 1
                else:
                    bad = True
    served, lengths, stop = [], [], False
    for r in range(R):
        want = max(pages(after[r]) - pages(max(cached[r], 0)), 0) if fits[r] else 0
        ok = fits[r]
        if want and (stop or want > count):
            ok, stop = False, True
        elif want:
            for j in range(pages(cached[r]), pages(after[r])):
                count -= 1
                table[r, j] = free[count]
        served.append(ok)
        lengths.append(after[r] if ok else cached[r])
    start = np.concatenate([[0], np.cumsum([max(a, 0) for a in added])]).astype(np.int64)
    slots, pos = np.full(tokens, -1, np.int64), np.zeros(tokens, np.int32)
    for r in range(R):
        for i in range(max(added[r], 0)):
            t, p = start[r] + i, cached[r] + i
            if t >= tokens:
                bad = True
                continue
            pos[t] = p
            if served[r]:
                slots[t] = int(table[r, p // page]) * page + p % page
    return table, free, count, np.array(lengths, np.int32), start.astype(np.int32), slots, pos, bad


def rope(x, pos, freq, axis, interleaved, inverse):
    """x float64 [T, H, D]; pos [axes, T]; freq float64 [P]; axis [P]."""
    x = x.copy()
    P = len(freq)
    for i in range(P):
        if not 0 <= axis[i] < pos.shape[0]:
            continue
        th = pos[axis[i]].astype(np.float64) * freq[i] * (-1 if inverse else 1)
        c, s = np.cos(th)[:, None], np.sin(th)[:, None]
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + P)
        a, b = x[:, :, ia].copy(), x[:, :, ib].copy()
        x[:, :, ia], x[:, :, ib] = a * c - b * s, b * c + a * s
    return x


def cache_bytes(codes, scales, fmt, D, page, pages, heads, rows):
    """Places of the cache's bytes: codes uint8 [tokens, heads, D/2] and scales
    [tokens, heads, n] (E8M0 bytes or uint32 words), token t at slot rows[t].
    Returns {flat byte index: value} for codes of K, of V and for scales."""
    kc, vc, sc = {}, {}, {}
    sb = np.ascontiguousarray(scales).view(np.uint8).reshape(scales.shape[0], scales.shape[1], -1)
    for t, slot in enumerate(rows):
        if not 0 <= slot < pages * page:
            continue
        pg, tok = divmod(int(slot), page)
        for h in range(heads):
            ph = pg * heads + h
            for e in range(0, D, 2):
                b, c, j = e // 32, e % 32 // 8, e % 8 // 2
                kc[ph * page * D // 2 + tok * D // 2 + (c * (D // 32) + b) * 4 + j] = codes[t, h, e // 2]
                g, w = divmod(e, D // 8)
                i, hh, cc, jj = tok // 16, tok // 8 % 2, tok // 2 % 4, tok % 2
                at = (((((ph * (page // 16) + i) * 2 + hh) * 8 + g) * 4 + cc) * 2 + jj) * (D // 16) + w // 2
                vc[at] = codes[t, h, e // 2]
            for j in range(sb.shape[2]):
                sc[(ph * page + tok) * sb.shape[2] + j] = sb[t, h, j]
    return kc, vc, sc


def attention(q, keys, values, start, lens, scale, window):
    """q float64 [T, Hq, D]; keys, values: per request float64 [L, H, D].
    Returns (o float64 [T, Hq, D], lse float64 [T, Hq])."""
    T, Hq, D = q.shape
    o, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    for r, (k, v) in enumerate(zip(keys, values)):
        n, L = start[r + 1] - start[r], int(lens[r])
        G = Hq // k.shape[1]
        for i in range(n):
            p = L - n + i
            lo = max(0, p - window + 1) if window else 0
            if p < lo:
                continue
            for h in range(Hq):
                s = k[lo:p + 1, h // G] @ q[start[r] + i, h] * scale
                m = s.max()
                e = np.exp(s - m)
                o[start[r] + i, h] = (e / e.sum()) @ v[lo:p + 1, h // G]
                lse[start[r] + i, h] = m + np.log(e.sum())
    return o, lse
