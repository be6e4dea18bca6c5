"""llma_attend_paged on bf16 rows loses no more than the output's own rounding: probabilities that keep 16 (steps) or 11 (tiles and many rows) significant bits, against the plain numpy
form in 64 bits; and what fp16 depends on: the scales of V's pages, far apart and in any order, values below fp16's normal range, probabilities far below the largest."""
import numpy as np
import pytest
import torch

import paged_oracle as oracle
from test_gpu_paged import attend_case, cache_values, i32, llma  # noqa: F401

pytestmark = pytest.mark.gpu


def check(llma, c, q, table, slots, lens, off, scale, p_err, least):  # noqa: F811
    """p_err: a probability's relative rounding; least: and its absolute one, relative to the row's largest"""
    D = q.shape[2]
    kv, vv, ks, vs = cache_values(c)
    V = vv * vs[..., None, None]
    want, size, big = oracle.attend(kv * ks[..., None, None], V, q.double().cpu().numpy(), table, slots, lens, off, scale, len(kv))
    got = llma.llma_attend_paged(c, q, i32(table), i32(lens), i32(off), int(np.diff(off).max()), scale, torch.zeros_like(q), slots=i32(slots)).double().cpu().numpy()
    # scores: D + 4 roundings of 2^-24 in products and sums, as much in the maximum's; exp2 and its argument 2^-20; a rounding per position in both sums; twice a
    # probability's (numerator and denominator); the output's own.  The absolute part: every position with the row's largest value
    p = 2 * (D + 4) * 2.0 ** -24 * big + 2.0 ** -20 + 2 * p_err + 2 * max(lens) * 2.0 ** -24
    seen = np.zeros_like(want)
    for b in range(len(lens)):
        pages = [int(x) for x in table[slots[b], :(lens[b] + 63) // 64]]
        v = np.abs(V[pages]).transpose(1, 0, 2, 3).reshape(V.shape[1], -1, D)[:, :lens[b]]
        top = np.maximum.accumulate(np.nan_to_num(v), axis=1)
        m = off[b + 1] - off[b]
        for j in range(m):
            n = lens[b] - m + j
            if n >= 0:
                seen[off[b] + j] = (n + 1) * np.repeat(top[:, n], q.shape[1] // V.shape[1], 0)
    tol = (1 + 2.0 ** -7) * (size * p[..., None] + least * seen) + 2.0 ** -8 * np.abs(want) + 1e-37
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - want) / tol)
    assert worst <= 1.0, worst


# steps of up to two tiles; of more, and many rows: one plane of fp16, whose half step at its bottom is 2^-25, where a row's largest is 2^15, or 2^7 and more
STEPS, TILES, ROWS = dict(p_err=2.0 ** -16, least=0.0), dict(p_err=2.0 ** -11, least=2.0 ** -40), dict(p_err=2.0 ** -11, least=2.0 ** -32)


def is_rows(q, lens, rows, kv):
    r = max(rows) * (q.shape[1] // kv)
    return r > 64 and min(len(rows) * -(-r // 128), len(q) * (q.shape[1] // kv) // 128 + len(rows)) * kv >= 160


@pytest.mark.parametrize("D,heads,kv,lens,rows", [
    (64, 8, 8, [1001], [1]), (128, 32, 32, [700, 65], [9, 9]), (128, 4, 1, [5, 900, 64, 70, 3000, 1], [3, 9, 9, 1, 5, 1]),
    (64, 12, 2, [3000, 40], [7, 8]), (128, 6, 2, [300, 2700], [33, 20]), (128, 2, 1, [9000], [1]), (64, 8, 8, [500, 300], [500, 40])])
def test_steps(llma, D, heads, kv, lens, rows):  # noqa: F811
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, "bf16", 31 + D + heads)
    assert not is_rows(q, lens, rows, kv)
    check(llma, c, q, table, slots, lens, off, D ** -0.5, **(TILES if max(rows) * (heads // kv) > 32 else STEPS))


@pytest.mark.parametrize("D,heads,kv,lens,rows", [(64, 64, 64, [330], [300]), (128, 96, 32, [200, 450], [60, 140]), (64, 40, 40, [2300], [500])])
def test_many_rows(llma, D, heads, kv, lens, rows):  # noqa: F811
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, "bf16", 33 + D + heads)
    assert is_rows(q, lens, rows, kv)
    check(llma, c, q, table, slots, lens, off, D ** -0.5, **ROWS)


@pytest.mark.parametrize("H", [40, 6])
@pytest.mark.parametrize("name,exponents", [
    ("rising", [-60, -30, -12, -3, 0, 5, 14, 40, 70]), ("falling", [70, 40, 14, 5, 0, -3, -12, -30, -60]), ("edges", [0, 7, -8, 0, -15, 0, 8, -8, -23]),
    ("zeros between", [20, None, 13, None, None, 28, 3, None, 20]), ("far", [-40, 60, -30, None, 60, -40, -40, 60, -40]), ("tiny", [-64] * 9)])
def test_scales_of_pages(llma, name, exponents, H):  # noqa: F811
    """a page's V as large as 448 * 2^exponent (None: zeros, whose scale is 2^-64); the causal rows of a prompt see one page more after every 64"""
    lens, rows, D = [64 * len(exponents) - 20], [64 * len(exponents) - 20], 64
    c, q, table, slots, off = attend_case(llma, lens, rows, H, H, D, "bf16", 41, q_size=1.0)
    assert is_rows(q, lens, rows, H) == (H == 40)                        # (many rows; tiles of 64 rows, the pages in shares or whole)
    for b, e in enumerate(exponents):
        page = int(table[slots[0], b])
        if e is None:
            c.v[page] = 0
        c.v_scale[page] = 2.0 ** (-64 if e is None else e)
    for t in (table, np.concatenate([table, np.full((len(table), 45 - table.shape[1]), -1)], 1)):
        check(llma, c, q, t, slots, lens, off, 0.125, **(ROWS if H == 40 else TILES))


@pytest.mark.parametrize("H", [80, 3])
def test_small_values_beside_large_scales(llma, H):  # noqa: F811
    """pages whose scale is 2^15 below the one before them, that one all zeros: the smallest codes, from an average over all rows"""
    lens, rows, D = [256], [256], 64
    c, q, table, slots, off = attend_case(llma, lens, rows, H, H, D, "bf16", 43)
    assert is_rows(q, lens, rows, H) == (H == 80)
    first, rest = int(table[slots[0], 0]), [int(p) for p in table[slots[0], 1:4]]
    c.v[first] = 0
    c.v_scale[first] = 1.0
    for p in rest:
        c.v[p] = torch.randint(0, 8, c.v[p].shape, device="cuda", dtype=torch.uint8)          # below e4m3's normal range
        c.v_scale[p] = 2.0 ** -15
    check(llma, c, q, table, slots, lens, off, 0.0, **(ROWS if H == 80 else TILES))


@pytest.mark.parametrize("H", [80, 4])
@pytest.mark.parametrize("below", [10, 17, 21, 24])
def test_probabilities_far_below_the_largest(llma, below, H):  # noqa: F811
    """one position takes nearly all of every row; its V is zero, what is left is the others' sum, 2^-below each"""
    lens, rows, D = [1500], [200], 64
    c, q, table, slots, off = attend_case(llma, lens, rows, H, H, D, "bf16", 47)
    assert is_rows(q, lens, rows, H) == (H == 80)
    used = [int(p) for p in table[slots[0], :24]]
    c.k[used] = 0
    c.v[used] &= 0x7F                                                    # (averages of positive numbers)
    c.k[used[3], :, 7, 0] = 0x38                                         # 1
    c.v[used[3], :, :, 7] = 0
    c.k_scale[used] = 1.0
    q.zero_()
    q[:, :, 0] = 1.0
    check(llma, c, q, table, slots, lens, off, below * float(np.log(2.0)), **(ROWS if H == 80 else TILES))
