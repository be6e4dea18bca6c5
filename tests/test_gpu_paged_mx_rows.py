"""Attention over 4-bit pages in its form for many rows: what rows, slots, pages and scales can be, at sizes that take that form.  Each test looks at the list of row blocks' pages that the
form leaves at the start of its workspace, so that another rule for which calls take it cannot turn the test into one of the steps' form."""
import numpy as np
import pytest
import torch

from test_gpu_paged_mx import DT, HALF, PAGE, attend_case, cached, check_attend, i32, llma, random_cache  # noqa: F401

pytestmark = pytest.mark.gpu


def block_list(lens, rows, group, dtype):
    """pages before every block of rows, as many blocks a sequence as the longest has, and of all: a block has the pages that its last row sees, one if that is none"""
    per = 64 if dtype == "fp32" else 128
    blocks = -(-max(rows) * group // per)
    assert blocks > 1                                                   # (of one block the list is the steps' list of sequences)
    pages = []
    for n, m in zip(lens, rows):
        for r0 in range(0, blocks * per, per):
            furthest = n - m + (min(r0 + per, m * group) - 1) // group
            pages.append(0 if r0 >= m * group else 1 if furthest < 0 else furthest // PAGE + 1)
    return np.concatenate([[0], np.cumsum(pages)])


class Work:
    """a workspace of the size asked for, and whether the call that used it took the form for many rows"""

    def __init__(self, llma, lens, rows, q, c, table, dtype):  # noqa: F811
        heads, D, kv = q.shape[1], q.shape[2], c.k.shape[1]
        self.size = llma.llma_attend_paged_mx_workspace(len(lens), table.shape[1], heads, kv, D, max(rows))
        self.ints = torch.full((self.size // 4,), -1, dtype=torch.int32, device="cuda")
        self.want = block_list(lens, rows, heads // kv, dtype)

    def check(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.ints[:len(self.want)].cpu().numpy(), self.want)
        self.ints.fill_(-1)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("D,heads,kv", [(128, 4, 2), (64, 8, 4)])
def test_rows_that_see_nothing(llma, dtype, D, heads, kv):  # noqa: F811
    """more rows than positions (the first of them come before the cache), empty sequences, sequences without positions, a page whose number is none: zeros there"""
    lens, rows = [2, 0, 0, 300], [200, 0, 100, 70]
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 51)
    table[slots[3], 1] = len(c.k) + 1
    w = Work(llma, lens, rows, q, c, table, dtype)
    out = check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype, workspace=w.ints)
    w.check()
    assert not out[:198].any() and not out[200:300].any() and out[199].any()


@pytest.mark.parametrize("D,heads,kv", [(128, 4, 2), (64, 16, 8)])
def test_slots_that_do_not_exist(llma, D, heads, kv):  # noqa: F811
    """sequences whose slot is none see nothing: zeros; the others are as without them"""
    rows, lens = [100] * 3, [200] * 3
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, "bf16", 95)
    w = Work(llma, lens, rows, q, c, table, "bf16")
    args = (i32(lens), i32(off), 100, 0.125)
    clean = llma.llma_attend_paged_mx(c, q, i32(table), *args, torch.empty_like(q), slots=i32(slots), workspace=w.ints)
    w.check()
    for bad in (-1, 3, 2 ** 31 - 1, -2 ** 31):
        got = llma.llma_attend_paged_mx(c, q, i32(table), *args, torch.full_like(q, 7.0), slots=i32([slots[0], bad, slots[2]]), workspace=w.ints)
        assert not got[100:200].any()
        for a in (0, 200):                                              # (cut elsewhere)
            assert (got[a:a + 100].float() - clean[a:a + 100].float()).abs().max() <= 2.0 ** -6 * clean.float().abs().max()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("D,heads,kv,rows", [(128, 4, 2, 100), (128, 4, 2, 700), (64, 48, 24, 100), (64, 10, 5, 700)])
def test_nan_stays_in_rows_that_see_it(llma, dtype, D, heads, kv, rows):  # noqa: F811
    """a NaN block of the last row's V: its 32 features of that row; of its K: all of that row; an early one of V: those of all rows"""
    lens, at, G = [rows + 35], rows + 34, heads // kv
    c, q, table, slots, off = attend_case(llma, lens, [rows], heads, kv, D, dtype, 61)
    w = Work(llma, lens, [rows], q, c, table, dtype)
    args = (i32(table), i32(lens), i32(off), rows, 0.125)
    attend = lambda: llma.llma_attend_paged_mx(c, q, *args, torch.empty_like(q), slots=i32(slots), workspace=w.ints)
    clean = attend()
    w.check()
    assert not clean.isnan().any()
    page, first = int(table[slots[0], at // PAGE]), int(table[slots[0], 0])
    for scale, p, pos, row, features in ((c.v_scale, page, at % PAGE, slice(rows - 1, rows), slice(32, 64)), (c.k_scale, page, at % PAGE, slice(rows - 1, rows), slice(0, D)),
                                         (c.v_scale, first, 2, slice(0, rows), slice(32, 64))):
        was = scale[p, 1, 1, pos].clone()
        scale[p, 1, 1, pos] = 255
        got, want = attend(), torch.zeros_like(q, dtype=torch.bool)
        want[row, G:2 * G, features] = True
        assert torch.equal(got.isnan(), want)
        assert torch.equal(got[~want], clean[~want])
        scale[p, 1, 1, pos] = was
    assert torch.equal(attend(), clean)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("D,heads,kv", [(128, 4, 4), (64, 32, 32)])
@pytest.mark.parametrize("shift,spread", [(0, 34), (-40, 3), (30, 3), (-22, 6), (11, 2)])
def test_scales_far_from_one(llma, dtype, D, heads, kv, shift, spread):  # noqa: F811
    """caches whose scales fp16 does not hold, or not all of them: small and large values of K and V, with queries and outputs in their types' range"""
    rows = 130
    c, q, table, slots, off = attend_case(llma, [300], [rows], heads, kv, D, dtype, 101)
    rng = np.random.default_rng(7)
    for s in (c.k_scale, c.v_scale):
        r = torch.tensor(rng.integers(-spread, 1, s.shape), device="cuda")
        by = shift if s is c.k_scale or dtype != "fp16" else max(min(shift, 8), -16)        # (fp16 outputs end at 65504, and lose bits below 2^-14)
        s.copy_(torch.where(s == 255, 255, s.int() + by + r).to(torch.uint8))
    w = Work(llma, [300], [rows], q, c, table, dtype)
    check_attend(llma, c, q, table, slots, [300], off, rows, dtype, scale=2.0 ** -(shift + 3), workspace=w.ints)
    w.check()


@pytest.mark.parametrize("D,heads,kv", [(128, 4, 2), (64, 48, 24)])
def test_subnormal_queries(llma, D, heads, kv):  # noqa: F811
    """fp16 queries below its normal range"""
    c, q, table, slots, off = attend_case(llma, [300], [130], heads, kv, D, "fp16", 103, q_size=4e-6)
    w = Work(llma, [300], [130], q, c, table, "fp16")
    check_attend(llma, c, q, table, slots, [300], off, 130, "fp16", scale=3e4, workspace=w.ints)
    w.check()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("lens,rows,D,heads,kv", [([2500], [70], 64, 64, 32), ([1500, 1, 0, 600], [130, 1, 0, 300], 64, 14, 7)])
def test_blocks_of_rows_in_several_shares(llma, dtype, lens, rows, D, heads, kv):  # noqa: F811
    """row blocks of head_dim 64 cut between workgroups"""
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 91, n_slots=len(lens) + 2, spare_rows=1)
    w = Work(llma, lens, rows, q, c, table, dtype)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype, workspace=w.ints)
    w.check()


# ------------------------------------------------------------------------------------------------ long sequences in one share
def long_case(llma, lens, rows, kv, D, dtype, seed):  # noqa: F811
    """as many query as key heads; pages of all sequences in a random order, some of them none"""
    rng = np.random.default_rng(seed)
    need = [(n + PAGE - 1) // PAGE for n in lens]
    P, blocks = sum(need), max(need)
    c = random_cache(llma, P, kv, D, seed, nans=False)
    perm, table = rng.permutation(P), np.full((len(lens), blocks), -1)
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b + 1])]
    table[0, [3, need[0] // 2]] = -1, P
    off = np.concatenate([[0], np.cumsum(rows)])
    q = torch.tensor(0.02 * rng.standard_normal((off[-1], kv, D)), dtype=torch.float32).to(DT[dtype]).cuda()
    return c, q, table, off


def check_heads(got, c, q, table, lens, off, dtype, heads):
    """some heads against 64 bits; tolerances as where all of a call is compared"""
    part = type(c)(*(t[:, heads].contiguous() for t in (c.k, c.v, c.k_scale, c.v_scale)))
    kv, vv = cached(part)
    D = q.shape[2]
    x, y = q[:, heads].double().cpu().numpy(), got[:, heads].double().cpu().numpy()
    for b, n in enumerate(lens):
        m = off[b + 1] - off[b]
        pages = table[b, :(n + PAGE - 1) // PAGE]
        have = ((pages >= 0) & (pages < len(kv))).repeat(PAGE)[:n]
        idx = np.where((pages >= 0) & (pages < len(kv)), pages, 0)
        sees = have[None] & (np.arange(n)[None] <= n - m + np.arange(m)[:, None])
        for h in range(len(heads)):
            K, V = (a[idx, h].reshape(-1, D)[:n] for a in (kv, vv))
            Q = x[off[b]:off[b + 1], h]
            s = np.where(sees, Q @ K.T * D ** -0.5, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            want, size = p @ V, p @ np.abs(V)
            big = np.where(sees, np.abs(Q) @ np.abs(K).T, 0).max(1) * D ** -0.5
            p_err = 2 * (D + 4) * 2.0 ** -24 * big + 2.0 ** -20 + {"bf16": 2.0 ** -11, "fp16": 2.0 ** -16, "fp32": 2.0 ** -24}[dtype]
            tol = (1 + 2.0 ** -7) * size * (p_err + 2 * n * 2.0 ** -24)[:, None] + HALF[dtype] * np.abs(want) + (2.0 ** -25 if dtype == "fp16" else 1e-30)
            worst = (np.abs(y[off[b]:off[b + 1], h] - want) / tol).max()
            assert worst <= 1.0, (b, heads[h], worst)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kv,D,lens,rows", [(512, 64, [64 * 200 + 1], [140]), (256, 128, [64 * 300 + 5], [300]), (512, 64, [64 * 66, 64 * 131 + 9], [140, 131])])
def test_blocks_of_many_rows_over_long_sequences(llma, dtype, kv, D, lens, rows):  # noqa: F811
    """a share has more than 128 pages of a block, whose page numbers come 64 at a time: with one share a key head from the block's first page on, with two also from a page inside"""
    c, q, table, off = long_case(llma, lens, rows, kv, D, dtype, 141)
    w = Work(llma, lens, rows, q, c, table, dtype)
    got = llma.llma_attend_paged_mx(c, q, i32(table), i32(lens), i32(off), max(rows), D ** -0.5, torch.full_like(q, 7.0), workspace=w.ints)
    w.check()
    assert (w.size < 1 << 16) == (kv == 512)                            # (parts only where a key head has two shares)
    check_heads(got, c, q, table, lens, off, dtype, [0, kv // 2 + 1, kv - 1])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kv,D,lens,rows", [(512, 64, [64 * 601 + 9], [3]), (512, 64, [64 * 270 + 5, 64 * 300], [3, 2]), (512, 64, [64 * 520 + 1], [30]), (512, 64, [64 * 300 + 2], [50]), (512, 128, [64 * 270], [1])])
def test_steps_over_long_sequences_in_one_share(llma, dtype, kv, D, lens, rows):  # noqa: F811
    """the steps' form with more than 256 pages of a sequence in a share, whose page numbers come 64 a wave at a time"""
    c, q, table, off = long_case(llma, lens, rows, kv, D, dtype, 143)
    size = llma.llma_attend_paged_mx_workspace(len(lens), table.shape[1], kv, kv, D, max(rows))
    assert size == 256                                                  # (no parts: a key head has one share)
    got = llma.llma_attend_paged_mx(c, q, i32(table), i32(lens), i32(off), max(rows), D ** -0.5, torch.full_like(q, 7.0))
    check_heads(got, c, q, table, lens, off, dtype, [0, kv // 2 + 1, kv - 1])
