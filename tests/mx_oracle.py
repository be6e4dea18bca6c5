"""Plain numpy forms, in 64 bits, of the 4-bit cache's calls and of token log probabilities (include/llma.h), for the tests of them."""
import numpy as np

PAGE, BLOCK = 64, 32
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([GRID, -GRID])


def exponent(amax):
    """of the smallest power of two s from 2^-64 to 2^120 with amax / s <= 7"""
    e = -64
    while amax > 7 * 2.0 ** e and e < 120:
        e += 1
    return e


def encode(x):
    """x [..., dh] float64: codes [..., dh] and scale bytes [..., dh / 32]"""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, BLOCK)
    finite = np.where(np.isfinite(b), np.abs(b), 0.0)
    e = np.vectorize(exponent, otypes=[int])(finite.max(-1))
    bad = np.isnan(b).any(-1)
    a = np.minimum(np.where(np.isnan(b), 0.0, np.abs(b)) / 2.0 ** e[..., None], 7.0)
    d = np.abs(a[..., None] - GRID)
    d = np.where(d == d.min(-1, keepdims=True), np.arange(8) % 2, 2)                       # ties to the even code
    codes = d.argmin(-1) | (np.signbit(b).astype(int) << 3)
    codes = np.where(bad[..., None], 0, codes)
    return codes.reshape(x.shape), np.where(bad, 255, e + 127)


def values(codes, scale):
    """what codes [..., dh] and scale bytes [..., dh / 32] stand for"""
    by = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (VALUES[codes].reshape(*scale.shape, BLOCK) * by[..., None]).reshape(codes.shape)


def unpack(pages, transposed):
    """bytes [pages, heads, 64, dh / 2] (or [pages, heads, dh / 2, 64]) as codes [pages, heads, 64, dh]"""
    c = pages.swapaxes(2, 3) if transposed else pages
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:3], 2 * c.shape[3]).astype(int)


def pack(codes, transposed):
    c = (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)
    return c.swapaxes(2, 3).copy() if transposed else c


def append(codes, scale, rows, slot_map):
    """codes [pages, heads, 64, dh] and scale [pages, heads, 64, dh / 32], changed in place; rows [n, heads, dh] float64"""
    c, s = encode(rows)
    for i, at in enumerate(slot_map):
        if 0 <= at < len(codes) * PAGE:
            codes[at // PAGE, :, at % PAGE], scale[at // PAGE, :, at % PAGE] = c[i], s[i]


def read(cached, table, slots, first, offsets, n_rows, n_pages, like):
    """cached [pages, heads, 64, dh] float64: rows [n_rows, heads, dh], `like` behind the last"""
    out = np.full((n_rows, *cached.shape[1:2], cached.shape[3]), like)
    for b in range(len(first)):
        for j in range(offsets[b + 1] - offsets[b]):
            if offsets[b] + j >= n_rows:
                break
            pos = first[b] + j
            page = table[slots[b], pos // PAGE] if 0 <= pos < PAGE * table.shape[1] and 0 <= slots[b] < len(table) else -1
            out[offsets[b] + j] = cached[page, :, pos % PAGE] if 0 <= page < n_pages else 0.0
    return out


def logprobs(x, token, temperature, n_top):
    """one row of logits, float64.  Returns logprob, rank, entropy, [tokens], [their logprobs]"""
    z = np.where(np.isnan(x), -np.inf, x)
    t = temperature if temperature > 0 else 1.0
    top = z.max()
    if top == -np.inf:
        lp = np.full_like(z, -np.inf)
        entropy = 0.0
    else:
        d = np.where(z == top, 0.0, z - (top if np.isfinite(top) else np.inf)) if np.isfinite(top) else np.where(z == top, 0.0, -np.inf)
        d = np.where(z == -np.inf, -np.inf, d / t if np.isfinite(t) else np.where(d == -np.inf, -np.inf, 0.0))
        lp = d - np.log(np.exp(d).sum())
        p = np.exp(lp)
        entropy = float(-(p[p > 0] * lp[p > 0]).sum())
    order = np.lexsort((np.arange(len(z)), -z))
    order = order[z[order] > -np.inf]
    tops = [int(v) for v in order[:n_top]]
    fill = n_top - len(tops)
    tops_lp = [float(lp[v]) for v in tops]
    given = 0 <= token < len(z)
    rank = int(((z > z[token]) | ((z == z[token]) & (np.arange(len(z)) < token))).sum()) if given else -1
    return (float(lp[token]) if given else -np.inf), rank, entropy, tops + [-1] * fill, tops_lp + [-np.inf] * fill
