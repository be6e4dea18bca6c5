"""Plain numpy forms, in 64 bits, of the stateless calls of serving on pages (include/llma.h), for the tests of them."""
import numpy as np

PAGE = 64


def e4m3_values():
    """what the 256 codes stand for: sign, four bits of exponent (bias 7), three of fraction; all ones: NaN"""
    v = np.empty(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v[c] = (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)) * (-1 if c & 128 else 1)
        if c & 127 == 127:
            v[c] = np.nan
    return v


VALUES = e4m3_values()


def to_e4m3(x):
    """the e4m3 value nearest to each x, ties to even, +-448 beyond it; NaN stays"""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    step = 2.0 ** (np.frexp(np.maximum(a, 2.0 ** -6))[1] - 1 - 3)
    return np.where(np.isnan(x), np.nan, np.sign(x) * np.round(a / step) * step)


def pow2_scale(amax):
    """the smallest power of two s from 2^-64 to 2^120 with amax / s <= 448"""
    s = 2.0 ** -64
    while amax / s > 448 and s < 2.0 ** 120:
        s *= 2
    return s


def append(values, scale, rows, slot_map):
    """values [pages, heads, 64, dh] (codes' values), scale [pages, heads]: changed in place.  rows [n, heads, dh] float64"""
    n, i = len(slot_map), 0
    while i < n:
        s = int(slot_map[i])
        if s < 0 or s // PAGE >= len(values):
            i += 1
            continue
        page, at, m = s // PAGE, s % PAGE, 1
        while i + m < n and slot_map[i + m] == s + m and at + m < PAGE:
            m += 1
        for h in range(values.shape[1]):
            x = rows[i:i + m, h]
            fin = np.abs(x[np.isfinite(x)])
            new = pow2_scale(fin.max() if fin.size else 0.0)
            if at > 0:
                new = max(new, scale[page, h])
                values[page, h, :at] = to_e4m3(values[page, h, :at] * (scale[page, h] / new))
            values[page, h, at:at + m] = to_e4m3(x / new)
            scale[page, h] = new
        i += m


def attend(k, v, q, table, slots, lens, offsets, scale, n_pages):
    """k, v [pages, heads, 64, dh] cached values; q [rows, query heads, dh].  Returns out, sum p |v| (both [rows, query heads, dh]) and
    max sum |q k| scale of each row and head, all zero for rows of no sequence"""
    out, size, big = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
    H, G = k.shape[1], q.shape[1] // k.shape[1]
    for b in range(len(lens)):
        slot = int(slots[b])
        m = int(offsets[b + 1] - offsets[b])
        n = int(lens[b])
        pages = [int(p) for p in table[slot, :(n + PAGE - 1) // PAGE]]
        have = np.array([0 <= p < n_pages for p in pages], bool).repeat(PAGE)[:n]
        idx = [p if 0 <= p < n_pages else 0 for p in pages]
        for h in range(H):
            K, V = (x[idx, h].reshape(-1, x.shape[-1])[:n] for x in (k, v))
            for j in range(m):
                see = have & (np.arange(n) <= n - m + j)
                if not see.any():
                    continue
                for g in range(G):
                    r, hq = int(offsets[b]) + j, h * G + g
                    s = K[see] @ q[r, hq] * scale
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[r, hq], size[r, hq] = p @ V[see], p @ np.abs(V[see])
                    big[r, hq] = (np.abs(K[see]) @ np.abs(q[r, hq])).max() * abs(scale)
    return out, size, big


def verify(logits, drafts, n_draft, probs, temperature, ua, us):
    """one sequence: logits [k + 1, V] float64, temperature a float.  Returns (accepted, next, [emitted], how near the nearest test came)"""
    kept, near = [], np.inf
    for j in range(n_draft + 1):
        z = np.where(np.isnan(logits[j]), -np.inf, logits[j])
        if z.max() == -np.inf:
            return len(kept), -1, kept + [-1], near
        if temperature > 0:
            top = z.max()
            p = np.exp(np.where(z == top, 0.0, np.where(z == top, 0.0, z) - np.where(z == top, 0.0, top)) / temperature)
            p /= p.sum()
        else:
            p = np.zeros_like(z)
            p[z.argmax()] = 1
        if j < n_draft:
            x = int(drafts[j])
            q = np.zeros_like(p)
            if 0 <= x < len(p):
                q[x] = 1
                if probs is not None and temperature > 0:
                    q = np.asarray(probs[j], np.float64)
                if temperature > 0 and p[x] > 0:                             # (otherwise whole numbers decide)
                    near = min(near, abs(float(ua[j]) * q[x] - p[x]) / p[x])
                if float(ua[j]) * q[x] < p[x]:
                    kept.append(x)
                    continue
            elif probs is not None and temperature > 0:
                q = np.asarray(probs[j], np.float64)
            w = np.maximum(p - q, 0)
            p = w if w.sum() > 0 else p
        c = np.cumsum(p)
        if temperature > 0:
            over = np.nonzero((c > float(us) * c[-1]) & (p > 0))[0]
            token = int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1])
        else:
            token = int(z.argmax())
        return len(kept), token, kept + [token], near
