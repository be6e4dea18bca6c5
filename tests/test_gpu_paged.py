"""Pages of 8-bit cache on the GPU: llma_map_pages, llma_append_paged and llma_attend_paged against plain numpy forms in 64 bits."""
import numpy as np
import pytest
import torch

import paged_oracle as oracle

pytestmark = pytest.mark.gpu
PAGE = 64
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}        # half a step of an output, relative


@pytest.fixture(scope="module")
def llma():
    import paper_2304_04487_amd as m
    m.load_library()
    return m


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ pages and slots
class Pages:
    """the definition, with lists; and the device's copy"""

    def __init__(self, llma, n_slots, blocks, n_pages, rng):
        self.llma, self.blocks, self.P = llma, blocks, n_pages
        self.free = [int(p) for p in rng.permutation(n_pages)]
        self.have = [[] for _ in range(n_slots)]
        self.dev = llma.PageTable.empty(n_slots, blocks, n_pages)
        self.dev.free_pages.copy_(i32(self.free))

    def step(self, slots, lens, rows, max_rows, named=True):
        """one call; returns what the device wrote and what the definition says"""
        B = len(slots)
        need = [(lens[s] + r + PAGE - 1) // PAGE for s, r in zip(slots, rows)]
        back = [(s, b) for s, n in zip(slots, need) for b in range(n, len(self.have[s]))]
        lack = sum(max(0, n - len(self.have[s])) for s, n in zip(slots, need)) - len(self.free) - len(back)
        status = max(lack, 0)
        if status == 0:
            for s, b in reversed(back):
                self.free.append(self.have[s].pop())
            for s, n in zip(slots, need):
                while len(self.have[s]) < n:
                    self.have[s].append(self.free.pop())
        live = [r if status == 0 else 0 for r in rows]
        off = np.concatenate([[0], np.cumsum(live)])
        slot_map, pos = np.full(max_rows, -1), np.zeros(max_rows, int)
        for b, s in enumerate(slots):
            for i in range(live[b]):
                p = lens[s] + i
                slot_map[off[b] + i], pos[off[b] + i] = self.have[s][p // PAGE] * PAGE + p % PAGE, p
        want = [off, [lens[s] + n for s, n in zip(slots, live)], slot_map, pos, [status]]
        got = [torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (B + 1, B, max_rows, max_rows, 1)]
        self.llma.llma_map_pages(self.dev, i32(lens), i32(rows), *got, slots=i32(slots) if named else None)
        return got, want

    def check(self, got, want):
        for g, w, name in zip(got, want, ("row_offsets", "lens_after", "slot_map", "row_pos", "status")):
            assert g.cpu().tolist() == list(w), name
        assert self.dev.n_free.item() == len(self.free)
        assert self.dev.free_pages.cpu().tolist()[:len(self.free)] == self.free
        assert self.dev.owned.cpu().tolist() == [len(h) for h in self.have]
        table = self.dev.table.cpu().tolist()
        for h, t in zip(self.have, table):
            assert t == h + [-1] * (self.blocks - len(h))


@pytest.mark.parametrize("n_slots,blocks,named", [(1, 1, False), (3, 5, True), (70, 9, True), (1030, 3, True), (2500, 2, False)])
def test_map_pages_over_several_steps(llma, n_slots, blocks, named):
    """grants, returns, sequences that finish, steps of a part of the slots in any order; three steps on one state"""
    rng = np.random.default_rng(n_slots)
    pages = Pages(llma, n_slots, blocks, n_slots * blocks, rng)
    lens = [0] * n_slots
    for step in range(4):
        slots = list(range(n_slots)) if not named else [int(s) for s in rng.permutation(n_slots)[:max(1, n_slots - step)]]
        if step == 2:
            for s in slots[::3]:
                lens[s] = 0                                    # finished: gives all back unless it starts again
        rows = [int(rng.integers(0, min(150, blocks * PAGE - lens[s]) + 1)) for s in slots]
        got, want = pages.step(slots, lens, rows, sum(rows) + 5, named)
        pages.check(got, want)
        for s, r in zip(slots, rows):
            lens[s] = max(0, lens[s] + int(rng.integers(0, r + 1)) - int(rng.integers(0, 3)))


def test_map_pages_rows_in_a_launch_of_their_own(llma):
    rng = np.random.default_rng(5)
    pages = Pages(llma, 40, 40, 1600, rng)
    lens = [int(x) for x in rng.integers(0, 500, 40)]
    pages.check(*pages.step(list(range(40)), lens, [0] * 40, 3))
    rows = [int(x) for x in rng.integers(0, 1200, 40)]
    pages.check(*pages.step(list(range(40)), lens, rows, sum(rows) + 100))


def test_map_pages_taken_back_grants_leave_the_stack_as_it_was(llma):
    rng = np.random.default_rng(6)
    pages = Pages(llma, 9, 20, 180, rng)
    lens = [int(x) for x in rng.integers(1, 600, 9)]
    pages.check(*pages.step(list(range(9)), lens, [0] * 9, 0))
    before = pages.dev.free_pages.clone()
    pages.check(*pages.step(list(range(9)), lens, [300] * 9, 2700))
    pages.check(*pages.step(list(range(9)), lens, [0] * 9, 0))
    assert torch.equal(before[:pages.dev.n_free.item()], pages.dev.free_pages[:pages.dev.n_free.item()])


def test_map_pages_without_enough_pages_changes_nothing(llma):
    rng = np.random.default_rng(7)
    pages = Pages(llma, 4, 8, 10, rng)
    lens = [0, 0, 0, 0]
    pages.check(*pages.step([0, 1], lens, [200, 64], 300))
    lens = [200, 64, 0, 0]
    got, want = pages.step([2, 0, 3], lens, [300, 1, 100], 420)        # five and two pages where five are left
    assert want[4][0] == 2
    pages.check(got, want)
    pages.check(*pages.step([2, 0], lens, [300, 1], 310))


@pytest.mark.parametrize("what", ["len", "row", "twice", "slot", "blocks", "rows", "owned", "stack", "top"])
def test_map_pages_refuses_lists_that_make_no_sense(llma, what):
    rng = np.random.default_rng(8)
    pages = Pages(llma, 4, 8, 32, rng)
    lens = [100, 10, 64, 0]
    pages.check(*pages.step([0, 1, 2], lens, [0, 0, 0], 0))
    slots, rows, cap, code = [0, 1, 2], [3, 4, 5], 20, llma.LLMA_E_INVAL
    if what == "len":
        lens = [100, -1, 64, 0]
    elif what == "row":
        rows = [3, -4, 5]
    elif what == "twice":
        slots = [0, 2, 2]
    elif what == "slot":
        slots, code = [0, 4, 2], llma.LLMA_E_RANGE
    elif what == "blocks":
        rows, cap, code = [3, 600, 5], 700, llma.LLMA_E_RANGE
    elif what == "rows":
        cap, code = 11, llma.LLMA_E_RANGE
    elif what == "owned":
        pages.dev.owned[1] = 9
    elif what == "stack":
        pages.dev.n_free.fill_(33)
    elif what == "top":
        pages.dev.n_free.fill_(-1)
    state = [t.clone() for t in (pages.dev.table, pages.dev.owned, pages.dev.free_pages, pages.dev.n_free)]
    got = [torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (4, 3, cap, cap, 1)]
    llma.llma_map_pages(pages.dev, i32(lens), i32(rows), *got, slots=i32(slots))
    assert got[4].item() == code
    assert got[0].cpu().tolist() == [0] * 4 and got[2].cpu().tolist() == [-1] * cap and got[3].cpu().tolist() == [0] * cap
    for a, b in zip(state, (pages.dev.table, pages.dev.owned, pages.dev.free_pages, pages.dev.n_free)):
        assert torch.equal(a, b)


def test_map_pages_does_not_hand_on_numbers_of_no_page(llma):
    """a free list that holds what is no page's number: the rows get no slot, also where the slot would wrap around 32 bits"""
    pages = Pages(llma, 2, 4, 8, np.random.default_rng(9))
    pages.dev.free_pages.copy_(i32([8, -3, 1 << 26, (1 << 26) + 1, 5, 1 << 30, 100, 3]))
    got = [torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (3, 2, 400, 400, 1)]
    llma.llma_map_pages(pages.dev, i32([0, 0]), i32([200, 190]), *got)
    assert got[4].item() == 0
    slots = got[2].cpu().numpy()
    granted = pages.dev.table.cpu().numpy()
    for b, (at, rows) in enumerate(((0, 200), (200, 190))):
        for i in range(rows):
            p = int(granted[b, i // PAGE])
            assert slots[at + i] == (p * PAGE + i % PAGE if 0 <= p < 8 else -1)


# ------------------------------------------------------------------------------------------------ the write
def random_cache(llma, P, H, D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = llma.PagedCache.empty(P, H, D)
    for t in (c.k, c.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))      # NaN codes among them
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.pow(2.0, torch.randint(-9, 4, t.shape, generator=g, device="cuda").cpu().double()).float().cuda())
    return c


def cache_values(c):
    """codes' values [pages, heads, 64, dh] of K and V, and the scales, float64"""
    return (oracle.VALUES[c.k.cpu().numpy()], oracle.VALUES[c.v.cpu().numpy()].swapaxes(2, 3).copy(), c.k_scale.cpu().numpy().astype(np.float64), c.v_scale.cpu().numpy().astype(np.float64))


RUNS = {
    "one": [(2, 0, 1)],
    "last": [(1, 63, 1)],
    "page": [(0, 0, 64)],
    "inside": [(4, 13, 30), (3, 5, 1), (0, 1, 2)],
    "step": [(p, o, n) for p, o, n in ((0, 60, 4), (1, 0, 5), (2, 17, 9), (4, 62, 2), (3, 0, 9), (5, 33, 31))],
    "over two windows": [(0, 50, 14), (1, 0, 64), (2, 0, 64), (3, 0, 7)],
}


@pytest.mark.parametrize("D,H", [(64, 1), (128, 3), (64, 8), (128, 32)])
@pytest.mark.parametrize("name", list(RUNS))
@pytest.mark.parametrize("dtype", list(DT))
def test_append_is_the_definition_bit_for_bit(llma, D, H, name, dtype):
    """scales, codes of the runs, codes before them and behind them; padding rows and rows whose page does not exist are skipped"""
    rng = np.random.default_rng(D * H + len(name))
    c = random_cache(llma, 6, H, D, 3)
    slot_map = [-1] + [p * PAGE + o + i for p, o, n in RUNS[name] for i in range(n)] + [-1, 6 * PAGE, 6 * PAGE + 1, 7 * PAGE + 3]
    rows = rng.standard_normal((len(slot_map), 2, H, D)) * np.exp2(rng.integers(-3, 5, (len(slot_map), 2, H, 1)))
    rows[:, :, :, 5] *= 1e-4                                            # (below the codes' normal range)
    rows[1, 0, 0, 3], rows[1, 1, 0, 1], rows[1, 0, 0, 7], rows[1, 1, 0, 9] = np.inf, -np.inf, np.nan, np.nan
    x = torch.tensor(rows).to(DT[dtype]).cuda()
    want = cache_values(c)
    exact = x.double().cpu().numpy()
    oracle.append(want[0], want[2], exact[:, 0], slot_map)
    oracle.append(want[1], want[3], exact[:, 1], slot_map)
    llma.llma_append_paged(c, x[:, 0], x[:, 1], i32(slot_map))
    got = cache_values(c)
    for g, w, part in zip(got, want, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(g, w, equal_nan=True), part
    # the same rows again: nothing changes
    llma.llma_append_paged(c, x[:, 0], x[:, 1], i32(slot_map))
    for g, w in zip(cache_values(c), got):
        assert np.array_equal(g, w, equal_nan=True)


def test_append_takes_any_strides_and_sizes_of_values(llma):
    """heads outermost, every second row of a wider buffer; values from 1e-30 to the largest fp32, zeros alone"""
    H, D, n = 4, 64, 70
    rng = np.random.default_rng(1)
    for big in (1e-30, 1e-9, 3.0, 1e20, 3.4e38, 0.0):
        c = random_cache(llma, 3, H, D, 5)
        buf = torch.tensor(rng.uniform(-1, 1, (H, 2 * n, 3 * D)) * big, dtype=torch.float32, device="cuda")
        k, v = buf[:, ::2, D:2 * D].transpose(0, 1), buf[:, 1::2, 2 * D:].transpose(0, 1)
        slot_map = list(range(PAGE, PAGE + n))
        want = cache_values(c)
        oracle.append(want[0], want[2], k.double().cpu().numpy(), slot_map)
        oracle.append(want[1], want[3], v.double().cpu().numpy(), slot_map)
        llma.llma_append_paged(c, k, v, i32(slot_map))
        for g, w in zip(cache_values(c), want):
            assert np.array_equal(g, w, equal_nan=True), big


# ------------------------------------------------------------------------------------------------ attention
def attend_case(llma, lens, rows, heads, kv, D, dtype, seed, n_slots=None, spare_rows=0, q_size=2.0):
    """a cache filled with normal values (positions behind a sequence's last: NaN codes), a table over it, queries"""
    rng = np.random.default_rng(seed)
    B = len(lens)
    n_slots = n_slots or B
    need = [(n + PAGE - 1) // PAGE for n in lens]
    P, blocks = sum(need) + 2, max(max(need), 1)
    perm = rng.permutation(P)
    slots = rng.permutation(n_slots)[:B]
    table = rng.integers(-5, P + 5, (n_slots, blocks))                  # what is not a sequence's page is anything
    at = 0
    for b in range(B):
        table[slots[b], :need[b]] = perm[at:at + need[b]]
        at += need[b]
    c = llma.PagedCache.empty(P, kv, D)
    k = rng.standard_normal((P, kv, PAGE, D)) * np.exp(0.5 * rng.standard_normal((1, kv, 1, D)))
    v = rng.standard_normal((P, kv, D, PAGE))
    for x, codes, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        s = np.vectorize(oracle.pow2_scale)(np.abs(x).max((2, 3)))
        codes.copy_(torch.tensor(x / s[..., None, None], dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8))
        scale.copy_(torch.tensor(s, dtype=torch.float32))
    for b in range(B):
        if lens[b] % PAGE:
            p = int(table[slots[b], need[b] - 1])
            c.k[p, :, lens[b] % PAGE:, :] = 0x7F
            c.v[p, :, :, lens[b] % PAGE:] = 0xFF
    off = np.concatenate([[0], np.cumsum(rows)])
    q = torch.tensor(rng.standard_normal((off[-1] + spare_rows, heads, D)) * q_size).to(DT[dtype]).cuda()
    return c, q, table, slots, off


def check_attend(llma, c, q, table, slots, lens, off, max_rows, dtype, out=None, scale=None, **kw):
    D = q.shape[2]
    scale = scale if scale is not None else D ** -0.5
    kv, vv, ks, vs = cache_values(c)
    want, size, big = oracle.attend(kv * ks[..., None, None], vv * vs[..., None, None], q.double().cpu().numpy(), table, slots, lens, off, scale, len(kv))
    if out is None:
        out = torch.full_like(q, 7.0)
    llma.llma_attend_paged(c, q, i32(table), i32(lens), i32(off), max_rows, scale, out, slots=i32(slots), **kw)
    got = out.double().cpu().numpy()
    n = off[-1]
    # A probability's relative error: D + 4 roundings of 2^-24 in its score's products and sums (relative to sum |q k| scale), as much again
    # from the maximum's score, a few in exp2 and its argument; and what its planes of bf16 leave: 2^-8 of itself (bf16), 2^-16, 2^-24.  Sums over
    # positions add a rounding each.  All of it times sum p |v|; then the output's own rounding.
    p_err = 2 * (D + 4) * 2.0 ** -24 * big + 2.0 ** -20 + {"bf16": 2.0 ** -8, "fp16": 2.0 ** -16, "fp32": 2.0 ** -24}[dtype]
    tol = (1 + 2.0 ** -7) * (size * (p_err + 2 * max(lens) * 2.0 ** -24)[..., None] if not np.isscalar(p_err) else 0) + HALF[dtype] * np.abs(want) + 1e-30
    if dtype == "fp16":
        tol = tol + 2.0 ** -25                                          # (half a step below fp16's normal range)
    assert np.isfinite(got[:n]).all()
    worst = np.max((np.abs(got[:n] - want[:n]) / tol[:n])) if n else 0.0
    assert worst <= 1.0, worst
    assert np.array_equal(got[n:], np.full_like(got[n:], 7.0))          # rows behind the last sequence
    return out


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("D,heads,kv", [(64, 8, 8), (128, 4, 1), (128, 6, 2), (64, 12, 2)])
@pytest.mark.parametrize("lens,rows", [
    ([1], [1]), ([64], [1]), ([65], [3]), ([1001], [1]), ([700], [9]), ([300], [33]), ([9], [9]),
    ([1, 64, 63, 130, 2, 257], [1, 1, 1, 1, 1, 1]),
    ([5, 900, 64, 70, 1500, 1], [3, 9, 9, 1, 5, 1]),
    ([40, 129, 3], [40, 100, 3]),
])
def test_attend_against_the_plain_form(llma, dtype, D, heads, kv, lens, rows):
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 11 + len(lens) + lens[0], n_slots=len(lens) + 3, spare_rows=2)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype)


@pytest.mark.parametrize("dtype", list(DT))
def test_attend_many_ragged_sequences(llma, dtype):
    rng = np.random.default_rng(21)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(2000), 300))]
    rows = [int(min(n, r)) for n, r in zip(lens, rng.integers(1, 6, 300))]
    c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, 64, dtype, 22, spare_rows=3)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_long_sequence_and_large_scores(llma, dtype):
    """one sequence in many shares; scores so large that one position takes all, and a scale of zero"""
    lens, rows = [9000], [2]
    for q_size, scale in ((2.0, None), (60.0, None), (1.0, 0.0), (1.0, -0.3)):
        c, q, table, slots, off = attend_case(llma, lens, rows, 2, 1, 128, dtype, 31, q_size=q_size)
        check_attend(llma, c, q, table, slots, lens, off, 2, dtype, scale=scale)


def test_attend_prompt_rows(llma):
    """hundreds of rows on top of a cache, several sequences, both head layouts"""
    for lens, rows, heads, kv, D in (([700, 260], [500, 260], 4, 2, 128), ([513], [513], 2, 2, 64), ([300, 40, 1000], [7, 40, 300], 8, 1, 64)):
        c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, "bf16", 41)
        check_attend(llma, c, q, table, slots, lens, off, max(rows), "bf16")


@pytest.mark.parametrize("rows", [[4, 0, 6, 9], [200, 0, 100, 70]])
def test_attend_rows_that_see_nothing(llma, rows):
    """more rows than positions (the first of them come before the cache), empty sequences, pages whose number is none: zeros there"""
    lens = [2, 0, 0, 300]
    c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, 64, "fp32", 51)
    table[slots[3], 1] = len(c.k) + 1
    out = check_attend(llma, c, q, table, slots, lens, off, max(rows), "fp32")
    assert not out[:rows[0] - 2].any() and not out[rows[0]:rows[0] + rows[2]].any() and out[rows[0] - 1].any()


@pytest.mark.parametrize("rows", [[3], [70]])
def test_attend_nan_stays_in_rows_that_see_it(llma, rows):
    """a NaN in the last row's V, in its K: only that row (and all of a NaN query's) become NaN"""
    lens = [100]
    for which in ("v", "k", "q"):
        c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, 64, "bf16", 61)
        clean = llma.llma_attend_paged(c, q, i32(table), i32(lens), i32(off), rows[0], 0.125, torch.empty_like(q), slots=i32(slots))
        page = int(table[slots[0], 1])
        if which == "v":
            c.v[page, 1, 5, 35] = 0x7F
        elif which == "k":
            c.k[page, 1, 35, 5] = 0x7F
        else:
            q[0, 3, 9] = float("nan")
        got = llma.llma_attend_paged(c, q, i32(table), i32(lens), i32(off), rows[0], 0.125, torch.empty_like(q), slots=i32(slots))
        want_nan = torch.zeros_like(q, dtype=torch.bool)
        if which == "v":
            want_nan[-1, 2:, 5] = True
        elif which == "k":
            want_nan[-1, 2:, :] = True
        else:
            want_nan[0, 3, :] = True
        assert torch.equal(got.isnan(), want_nan), which
        assert torch.equal(got[~want_nan], clean[~want_nan]), which


def test_attend_strides_workspace_and_streams(llma):
    """queries inside a wider projection, output with heads outermost, a workspace of the caller's, a side stream"""
    lens, rows, D = [400, 90], [9, 9], 64
    c, q, table, slots, off = attend_case(llma, lens, rows, 8, 4, D, "bf16", 71)
    wide = torch.zeros((18, 8 + 2 * 4, D), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = q
    out = torch.empty((8, 18, D), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    ws = torch.empty(llma.llma_attend_paged_workspace(2, table.shape[1], 8, 4, D, 9), dtype=torch.uint8, device="cuda")
    check_attend(llma, c, wide[:, :8], table, slots, lens, off, 9, "bf16", out=out.fill_(7.0), workspace=ws)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    args = (i32(table), i32(lens), i32(off))
    plain = llma.llma_attend_paged(c, q, *args, 9, 0.125, torch.empty_like(q), slots=i32(slots))
    s2, o2 = i32(slots), torch.empty_like(q)
    torch.cuda.synchronize()
    llma.llma_attend_paged(c, q, *args, 9, 0.125, o2, slots=s2, stream=st)
    st.synchronize()
    assert torch.equal(plain, o2)


@pytest.mark.parametrize("heads,kv,rows,most", [(8, 4, [9, 5], 6), (96, 96, [90, 70], 68)])
def test_attend_writes_max_rows_of_a_sequence_at_most(llma, heads, kv, rows, most):
    """what is written is what a call for all rows writes there; q that ends inside the last sequence likewise"""
    lens = [130, 75]
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, 64, "bf16", 73)
    args = (i32(table), i32(lens), i32(off))
    full = llma.llma_attend_paged(c, q, *args, max(rows), 0.125, torch.empty_like(q), slots=i32(slots))
    some = llma.llma_attend_paged(c, q, *args, most, 0.125, torch.full_like(q, 7.0), slots=i32(slots))
    for b in range(2):
        a, e = off[b], off[b + 1]
        m = min(most, rows[b])
        assert (some[a:a + m].float() - full[a:a + m].float()).abs().max() <= 2.0 ** -6 * full.float().abs().max()      # (another form may have computed it)
        assert (some[a + m:e] == 7.0).all()
    short = llma.llma_attend_paged(c, q[:off[1] + 2], *args, max(rows), 0.125, torch.full_like(q, 7.0)[:off[1] + 2], slots=i32(slots))
    assert (short.float() - full[:off[1] + 2].float()).abs().max() <= 2.0 ** -6 * full.float().abs().max()


def test_attend_pages_past_32_bits(llma):
    """pages whose bytes lie more than 2^32 behind the cache's start"""
    H, D = 8, 128
    P = (1 << 32) // (H * PAGE * D) + 40
    c = llma.PagedCache(torch.zeros((P, H, PAGE, D), dtype=torch.uint8, device="cuda"), torch.zeros((P, H, D, PAGE), dtype=torch.uint8, device="cuda"),
                        torch.ones((P, H), device="cuda"), torch.ones((P, H), device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((200, 2, H, D), generator=g, device="cuda").to(torch.bfloat16)
    far, near = [P - 1, P - 5, P - 2, P - 30], [3, 1, 0, 2]
    slot = lambda pages: i32([pages[i // PAGE] * PAGE + i % PAGE for i in range(200)])
    for pages in (far, near):
        llma.llma_append_paged(c, x[:, 0], x[:, 1], slot(pages))
    q = torch.randn((3, 16, D), generator=g, device="cuda").to(torch.bfloat16)
    a, b = (llma.llma_attend_paged(c, q, i32([pages]), i32([200]), i32([0, 3]), 3, 0.09, torch.empty_like(q)) for pages in (far, near))
    assert torch.equal(a, b) and a.float().abs().max() > 0.01
    assert torch.equal(c.k[far], c.k[near]) and torch.equal(c.v[far], c.v[near])


def test_a_step_of_all_of_them_together_captured_and_replayed(llma):
    """map, append and attend as a serving loop runs them, eagerly and as one graph replayed over growing sequences"""
    B, H, heads, D, m, blocks = 5, 2, 6, 64, 4, 6
    rng = np.random.default_rng(81)
    fresh = [i32([0] * B), i32([m] * B)]

    def state():
        pages = llma.PageTable.empty(B, blocks, B * blocks)
        cache = random_cache(llma, B * blocks, H, D, 9)
        bufs = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (B + 1, B, B * m, B * m, 1)]
        return pages, cache, bufs, torch.zeros(B, dtype=torch.int32, device="cuda"), torch.empty((B * m, heads + 2 * H, D), dtype=torch.bfloat16, device="cuda"), \
            torch.empty((B * m, heads, D), dtype=torch.bfloat16, device="cuda")

    def step(s):
        pages, cache, (off, after, slot_map, pos, status), lens, x, out = s
        llma.llma_map_pages(pages, lens, fresh[1], off, after, slot_map, pos, status)
        llma.llma_append_paged(cache, x[:, heads:heads + H], x[:, heads + H:], slot_map)
        llma.llma_attend_paged(cache, x[:, :heads], pages.table, after, off, m, D ** -0.5, out)

    eager, replayed = state(), state()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step(replayed)
    lens = np.zeros(B, int)
    k_all, v_all = [[] for _ in range(B)], [[] for _ in range(B)]
    for it in range(12):
        x = torch.tensor(rng.standard_normal(eager[4].shape), dtype=torch.bfloat16, device="cuda")
        for s in (eager, replayed):
            s[4].copy_(x)
            s[3].copy_(i32(lens))
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert eager[2][4].item() == 0
        assert torch.equal(eager[5], replayed[5])
        for a, b in zip((eager[0].table, eager[0].n_free, *eager[2]), (replayed[0].table, replayed[0].n_free, *replayed[2])):
            assert torch.equal(a, b)
        kv, vv, ks, vs = cache_values(eager[1])
        off = np.arange(B + 1) * m
        want, size, big = oracle.attend(kv * ks[..., None, None], vv * vs[..., None, None], x[:, :heads].double().cpu().numpy(), eager[0].table.cpu().numpy(), range(B), lens + m, off, D ** -0.5, B * blocks)
        tol = size * (2 * (D + 4) * 2.0 ** -24 * big + 2.0 ** -8 + 2.0 ** -12)[..., None] + 2.0 ** -8 * np.abs(want) + 1e-30
        assert (np.abs(eager[5].double().cpu().numpy() - want) <= tol).all()
        lens = lens + rng.integers(1, m + 1, B)                          # the accepted rows stay
        lens[rng.integers(0, B)] = 0                                     # one sequence ends, another begins in its place
        lens = np.minimum(lens, blocks * PAGE - m)
