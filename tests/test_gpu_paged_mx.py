"""Pages of 4-bit cache on the GPU: llma_append_paged_mx, llma_attend_paged_mx and llma_read_paged_mx, and llma_read_paged, against plain numpy forms in 64 bits."""
import numpy as np
import pytest
import torch

import mx_oracle as mx
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


def random_cache(llma, P, H, D, seed, nans=True):
    """any codes; scales from 2^-9 to 2^4, some that stand for NaN"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = llma.PagedMxCache.empty(P, H, D)
    for t in (c.k, c.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.randint(118, 132, t.shape, generator=g, device="cuda", dtype=torch.uint8))
        if nans:
            t.masked_fill_(torch.rand(t.shape, generator=g, device="cuda") < 0.02, 255)
    return c


def codes_of(c):
    """codes [pages, heads, 64, dh] of K and V, and their scale bytes [pages, heads, 64, dh / 32]"""
    k, v, ks, vs = (t.cpu().numpy() for t in (c.k, c.v, c.k_scale, c.v_scale))
    return mx.unpack(k, False), mx.unpack(v, True), ks.swapaxes(2, 3).astype(int), vs.swapaxes(2, 3).astype(int)


def cached(c):
    k, v, ks, vs = codes_of(c)
    return mx.values(k, ks), mx.values(v, vs)


# ------------------------------------------------------------------------------------------------ the write
RUNS = {
    "one": [(2, 0, 1)],
    "last": [(1, 63, 1)],
    "page": [(0, 0, 64)],
    "inside": [(4, 13, 30), (3, 5, 1), (0, 1, 2)],
    "step": [(p, o, n) for p, o, n in ((0, 60, 4), (1, 0, 5), (2, 17, 9), (4, 62, 2), (3, 0, 9), (5, 33, 31))],
    "over two windows": [(0, 50, 14), (1, 0, 64), (2, 0, 64), (3, 0, 7)],
    "any order": [(3, 9, 1), (3, 8, 1), (0, 4, 1), (3, 10, 3), (5, 40, 1), (0, 6, 1), (0, 5, 1), (1, 20, 4), (1, 16, 4), (2, 3, 5)],
}


@pytest.mark.parametrize("D,H", [(64, 1), (128, 3), (64, 8), (128, 32)])
@pytest.mark.parametrize("name", list(RUNS))
@pytest.mark.parametrize("dtype", list(DT))
def test_append_is_the_definition_bit_for_bit(llma, D, H, name, dtype):
    """codes and scales of the rows, nothing else; padding rows and rows whose page does not exist are skipped"""
    rng = np.random.default_rng(D * H + len(name))
    c = random_cache(llma, 6, H, D, 3)
    slot_map = [-1] + [p * PAGE + o + i for p, o, n in RUNS[name] for i in range(n)] + [-1, 6 * PAGE, 6 * PAGE + 1, 7 * PAGE + 3, -5]
    rows = rng.standard_normal((len(slot_map), 2, H, D)) * np.exp2(rng.integers(-3, 5, (len(slot_map), 2, H, 1)))
    rows[:, :, :, 5] *= 1e-4
    rows[:, :, :, 8:16] = np.array([7, 6, 5, 3.5, 2.5, -1.25, -0.25, 0.75])                # ties and the ends of the codes
    rows[1, 0, 0, 3], rows[1, 1, 0, 1], rows[1, 0, 0, 40], rows[1, 1, 0, 39] = np.inf, -np.inf, np.nan, np.nan
    x = torch.tensor(rows).to(DT[dtype]).cuda()
    want = codes_of(c)
    exact = x.double().cpu().numpy()
    mx.append(want[0], want[2], exact[:, 0], slot_map)
    mx.append(want[1], want[3], exact[:, 1], slot_map)
    llma.llma_append_paged_mx(c, x[:, 0], x[:, 1], i32(slot_map))
    for g, w, part in zip(codes_of(c), want, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(g, w), part


def test_append_takes_any_strides_and_sizes_of_values(llma):
    """heads outermost, every second row of a wider buffer; values from 1e-30 to the largest fp32, zeros alone"""
    H, D, n = 4, 64, 70
    rng = np.random.default_rng(1)
    for big in (1e-30, 1e-19, 1e-9, 3.0, 1e20, 3.4e38, 0.0):
        c = random_cache(llma, 3, H, D, 5)
        buf = torch.tensor(rng.uniform(-1, 1, (H, 2 * n, 3 * D)) * big, dtype=torch.float32, device="cuda")
        k, v = buf[:, ::2, D:2 * D].transpose(0, 1), buf[:, 1::2, 2 * D:].transpose(0, 1)
        slot_map = list(range(PAGE - 1, PAGE - 1 + n))
        want = codes_of(c)
        mx.append(want[0], want[2], k.double().cpu().numpy(), slot_map)
        mx.append(want[1], want[3], v.double().cpu().numpy(), slot_map)
        llma.llma_append_paged_mx(c, k, v, i32(slot_map))
        for g, w in zip(codes_of(c), want):
            assert np.array_equal(g, w), big


def test_append_of_prompts_at_every_alignment(llma):
    """runs of hundreds of rows that begin at each of a page's first positions, several in one call"""
    H, D, P = 2, 128, 24
    rng = np.random.default_rng(2)
    c = random_cache(llma, P, H, D, 6)
    slot_map, page = [], 0
    for begin in range(6):
        n = 150 + 7 * begin
        slot_map += [(page * PAGE) + begin + i for i in range(n)]
        page += (begin + n + PAGE - 1) // PAGE
    assert page <= P
    x = torch.tensor(rng.standard_normal((len(slot_map), 2, H, D)), dtype=torch.bfloat16, device="cuda")
    want = codes_of(c)
    mx.append(want[0], want[2], x[:, 0].double().cpu().numpy(), slot_map)
    mx.append(want[1], want[3], x[:, 1].double().cpu().numpy(), slot_map)
    llma.llma_append_paged_mx(c, x[:, 0], x[:, 1], i32(slot_map))
    for g, w in zip(codes_of(c), want):
        assert np.array_equal(g, w)


# ------------------------------------------------------------------------------------------------ rows out of the cache
def eight(llma, P, H, D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = llma.PagedCache.empty(P, H, D)
    for t in (c.k, c.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))      # NaN codes among them
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.tensor(np.exp2(np.random.default_rng(seed).integers(-9, 4, t.shape)), dtype=torch.float32))
    kv, vv = oracle.VALUES[c.k.cpu().numpy()], oracle.VALUES[c.v.cpu().numpy()].swapaxes(2, 3)
    return c, kv * c.k_scale.double().cpu().numpy()[..., None, None], vv * c.v_scale.double().cpu().numpy()[..., None, None]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("D,H", [(64, 1), (128, 3), (64, 5)])
@pytest.mark.parametrize("first,rows", [([0], [1]), ([63], [1]), ([0], [64]), ([5], [200]), ([0, 17, 64, 250], [3, 0, 130, 6]), ([200, 0, 1, 2, 3, 62], [400, 1, 1, 1, 1, 3])])
def test_read_is_the_definition(llma, bits, dtype, D, H, first, rows):
    """rounded once to the rows' type; head by head, and as rows inside wider ones; what lies behind the last row stays"""
    rng = np.random.default_rng(len(first) + D)
    P, blocks, B = 9, 8, len(first)
    if bits == 4:
        c = random_cache(llma, P, H, D, 13)
        kv, vv = cached(c)
    else:
        c, kv, vv = eight(llma, P, H, D, 13)
    table = rng.integers(-3, P + 3, (B + 2, blocks))                    # pages that are none among them
    slots = rng.permutation(B + 2)[:B]
    off = np.concatenate([[0], np.cumsum(rows)])
    n = off[-1] + 2
    k = torch.full((H, n, D), 7.0, dtype=DT[dtype], device="cuda").transpose(0, 1)
    v = torch.full((n, H, 2 * D), 7.0, dtype=DT[dtype], device="cuda")[:, :, D:]
    fn = llma.llma_read_paged_mx if bits == 4 else llma.llma_read_paged
    fn(c, i32(table), i32(first), i32(off), k, v, slots=i32(slots))
    for got, values in ((k, kv), (v, vv)):
        want = mx.read(values, table, slots, first, off, n, P, 7.0)
        assert torch.equal(got.cpu().isnan(), torch.tensor(want).isnan())
        assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(torch.tensor(want).to(DT[dtype])))


def test_read_defaults_and_lists_that_make_no_sense(llma):
    """no slots and no first; positions before the first and behind the table; offsets that fall, pass the rows, or begin late: nothing outside the rows is touched"""
    H, D, P, blocks = 2, 64, 4, 3
    c = random_cache(llma, P, H, D, 15)
    kv, vv = cached(c)
    table = np.array([[0, 1, 2], [3, 2, 1]])
    new = lambda n: [torch.full((n + 2, H, D), 7.0, device="cuda") for _ in range(2)]
    k, v = new(30)
    llma.llma_read_paged_mx(c, i32(table), None, i32([0, 20, 30]), k[:30], v[:30])
    for got, values in ((k, kv), (v, vv)):
        want = mx.read(values, table, [0, 1], [0, 0], [0, 20, 30], 32, P, 7.0)
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    for first, off, slots in (([-70, 150], [0, 100, 180], [0, 1]), ([0, 0], [0, 50, 500], [0, 1]), ([0, 0], [5, 40, 60], [1, 7]), ([0, 0], [0, 60, 20], [0, 1]),
                              ([2 ** 31 - 3, -2 ** 31], [0, 10, 20], [0, 1]), ([0, 0], [-2 ** 31, 2 ** 31 - 1, 3], [-1, 1])):
        k, v = new(180)
        llma.llma_read_paged_mx(c, i32(table), i32(first), i32(off), k[:180], v[:180], slots=i32(slots))
        torch.cuda.synchronize()
        assert (k[180:] == 7).all() and (v[180:] == 7).all() and (k[:max(0, off[0])] == 7).all()
        if off == sorted(off) and off[0] >= 0:
            want = mx.read(kv, table, slots, first, off, 180, P, 7.0)
            assert np.array_equal(k[:180].double().cpu().numpy(), want, equal_nan=True), (first, off)


# ------------------------------------------------------------------------------------------------ attention
def attend_case(llma, lens, rows, heads, kv, D, dtype, seed, n_slots=None, spare_rows=0, q_size=2.0, spread=0):
    """a cache filled with normal values (positions behind a sequence's last: scales that stand for NaN), a table over it, queries.  spread: blocks' sizes
    differ by up to 2^spread"""
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
    c = llma.PagedMxCache.empty(P, kv, D)
    k = rng.standard_normal((P, kv, PAGE, D)) * np.exp(0.5 * rng.standard_normal((1, kv, 1, D)))
    v = rng.standard_normal((P, kv, PAGE, D))
    for x, codes, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        n, s = mx.encode(x)
        s = s + rng.integers(-spread, 1, s.shape)
        codes.copy_(torch.tensor(mx.pack(n, codes is c.v)))
        scale.copy_(torch.tensor(s.swapaxes(2, 3).astype(np.uint8)))
    for b in range(B):
        if lens[b] % PAGE:
            p = int(table[slots[b], need[b] - 1])
            for s in (c.k_scale, c.v_scale):
                s[p, :, :, lens[b] % PAGE:] = 255
    off = np.concatenate([[0], np.cumsum(rows)])
    q = torch.tensor(rng.standard_normal((off[-1] + spare_rows, heads, D)) * q_size).to(DT[dtype]).cuda()
    return c, q, table, slots, off


def check_attend(llma, c, q, table, slots, lens, off, max_rows, dtype, out=None, scale=None, besides=None, **kw):
    D = q.shape[2]
    scale = scale if scale is not None else D ** -0.5
    kv, vv = cached(c)
    want, size, big = oracle.attend(kv, vv, q.double().cpu().numpy(), table, slots, lens, off, scale, len(kv))
    if out is None:
        out = torch.full_like(q, 7.0)
    llma.llma_attend_paged_mx(c, q, i32(table), i32(lens), i32(off), max_rows, scale, out, slots=i32(slots), **kw)
    got = out.double().cpu().numpy()
    n = off[-1]
    # A probability's relative error: D + 4 roundings of 2^-24 in its score's products and sums (relative to sum |q k| scale), as much again
    # from the maximum's score, a few in exp2 and its argument; and what the planes it enters the second product in leave: 2^-11 of itself (bf16 rows: one of fp16),
    # 2^-16, 2^-24.  Sums over positions add a rounding each.  All of it times sum p |v|; then the output's own rounding.
    p_err = 2 * (D + 4) * 2.0 ** -24 * big + 2.0 ** -20 + {"bf16": 2.0 ** -11, "fp16": 2.0 ** -16, "fp32": 2.0 ** -24}[dtype]
    tol = (1 + 2.0 ** -7) * size * (p_err + 2 * max(lens) * 2.0 ** -24)[..., None] + HALF[dtype] * np.abs(want) + 1e-30
    if dtype == "fp16":
        tol = tol + 2.0 ** -25                                          # (half a step below fp16's normal range)
    if besides is not None:
        tol[:n] += besides
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


@pytest.mark.parametrize("dtype", list(DT))
def test_attend_prompt_rows(llma, dtype):
    """hundreds of rows on top of a cache, several sequences, both head layouts"""
    for lens, rows, heads, kv, D in (([700, 260], [500, 260], 4, 2, 128), ([513], [513], 2, 2, 64), ([300, 40, 1000], [7, 40, 300], 8, 1, 64)):
        c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 41)
        check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows", [[3], [40], [130]])
def test_attend_blocks_of_different_sizes(llma, dtype, rows):
    """scales of neighbouring blocks and positions up to 2^20 apart"""
    c, q, table, slots, off = attend_case(llma, [300], rows, 4, 2, 128, dtype, 45, spread=20)
    check_attend(llma, c, q, table, slots, [300], off, max(rows), dtype)


@pytest.mark.parametrize("rows", [[4, 0, 6, 9], [200, 0, 100, 70]])
def test_attend_rows_that_see_nothing(llma, rows):
    """more rows than positions (the first of them come before the cache), empty sequences, pages whose number is none: zeros there"""
    lens = [2, 0, 0, 300]
    c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, 64, "fp32", 51)
    table[slots[3], 1] = len(c.k) + 1
    out = check_attend(llma, c, q, table, slots, lens, off, max(rows), "fp32")
    assert not out[:rows[0] - 2].any() and not out[rows[0]:rows[0] + rows[2]].any() and out[rows[0] - 1].any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [[3], [70], [700]])
def test_attend_nan_stays_in_rows_that_see_it(llma, rows, D):
    """a NaN block of the last row's V: its 32 features of that row; of its K: all of that row; of a query: all of the query's"""
    lens = [rows[0] + 35]
    at = lens[0] - 1
    for which in ("v", "k", "q"):
        c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, D, "bf16", 61)
        args = (i32(table), i32(lens), i32(off), rows[0], 0.125)
        clean = llma.llma_attend_paged_mx(c, q, *args, torch.empty_like(q), slots=i32(slots))
        page = int(table[slots[0], at // PAGE])
        if which == "v":
            c.v_scale[page, 1, 1, at % PAGE] = 255
        elif which == "k":
            c.k_scale[page, 1, 1, at % PAGE] = 255
        else:
            q[0, 3, 9] = float("nan")
        got = llma.llma_attend_paged_mx(c, q, *args, torch.empty_like(q), slots=i32(slots))
        want_nan = torch.zeros_like(q, dtype=torch.bool)
        if which == "v":
            want_nan[-1, 2:, 32:64] = True
        elif which == "k":
            want_nan[-1, 2:, :] = True
        else:
            want_nan[0, 3, :] = True
        assert torch.equal(got.isnan(), want_nan), which
        assert torch.equal(got[~want_nan], clean[~want_nan]), which
    # an early one, which all rows see
    c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, D, "bf16", 61)
    c.v_scale[int(table[slots[0], 0]), 0, 0, 2] = 255
    got = llma.llma_attend_paged_mx(c, q, *args, torch.empty_like(q), slots=i32(slots))
    assert got[:, :2, :32].isnan().all() and not got[:, :2, 32:].isnan().any() and not got[:, 2:].isnan().any()


def test_attend_strides_workspace_and_streams(llma):
    """queries inside a wider projection, output with heads outermost, a workspace of the caller's, a side stream"""
    lens, rows, D = [400, 90], [9, 9], 64
    c, q, table, slots, off = attend_case(llma, lens, rows, 8, 4, D, "bf16", 71)
    wide = torch.zeros((18, 8 + 2 * 4, D), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = q
    out = torch.empty((8, 18, D), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    ws = torch.empty(llma.llma_attend_paged_mx_workspace(2, table.shape[1], 8, 4, D, 9), dtype=torch.uint8, device="cuda")
    check_attend(llma, c, wide[:, :8], table, slots, lens, off, 9, "bf16", out=out.fill_(7.0), workspace=ws)
    st = torch.cuda.Stream()
    args = (i32(table), i32(lens), i32(off))
    plain = llma.llma_attend_paged_mx(c, q, *args, 9, 0.125, torch.empty_like(q), slots=i32(slots))
    s2, o2 = i32(slots), torch.empty_like(q)
    torch.cuda.synchronize()
    llma.llma_attend_paged_mx(c, q, *args, 9, 0.125, o2, slots=s2, stream=st)
    st.synchronize()
    assert torch.equal(plain, o2)


@pytest.mark.parametrize("heads,kv,rows,most", [(8, 4, [9, 5], 6), (96, 96, [90, 70], 68)])
def test_attend_writes_max_rows_of_a_sequence_at_most(llma, heads, kv, rows, most):
    """what is written is what a call for all rows writes there; q that ends inside the last sequence likewise"""
    lens = [130, 75]
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, 64, "bf16", 73)
    args = (i32(table), i32(lens), i32(off))
    full = llma.llma_attend_paged_mx(c, q, *args, max(rows), 0.125, torch.empty_like(q), slots=i32(slots))
    some = llma.llma_attend_paged_mx(c, q, *args, most, 0.125, torch.full_like(q, 7.0), slots=i32(slots))
    for b in range(2):
        a, e = off[b], off[b + 1]
        m = min(most, rows[b])
        assert (some[a:a + m].float() - full[a:a + m].float()).abs().max() <= 2.0 ** -6 * full.float().abs().max()      # (another form may have computed it)
        assert (some[a + m:e] == 7.0).all()
    short = llma.llma_attend_paged_mx(c, q[:off[1] + 2], *args, max(rows), 0.125, torch.full_like(q, 7.0)[:off[1] + 2], slots=i32(slots))
    assert (short.float() - full[:off[1] + 2].float()).abs().max() <= 2.0 ** -6 * full.float().abs().max()


def test_pages_past_32_bits(llma):
    """pages whose bytes lie more than 2^32 behind the cache's start: written, attended over, read back"""
    H, D = 8, 128
    P = (1 << 32) // (H * PAGE * D // 2) + 40
    c = llma.PagedMxCache(torch.zeros((P, H, PAGE, D // 2), dtype=torch.uint8, device="cuda"), torch.zeros((P, H, D // 2, PAGE), dtype=torch.uint8, device="cuda"),
                          *(torch.zeros((P, H, D // 32, PAGE), dtype=torch.uint8, device="cuda") for _ in range(2)))
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((200, 2, H, D), generator=g, device="cuda").to(torch.bfloat16)
    far, near = [P - 1, P - 5, P - 2, P - 30], [3, 1, 0, 2]
    slot = lambda pages: i32([pages[i // PAGE] * PAGE + i % PAGE for i in range(200)])
    for pages in (far, near):
        llma.llma_append_paged_mx(c, x[:, 0], x[:, 1], slot(pages))
    for part in (c.k, c.v, c.k_scale, c.v_scale):
        assert torch.equal(part[far], part[near]) and part[far].any()
    q = torch.randn((100, 16, D), generator=g, device="cuda").to(torch.bfloat16)
    for m in (3, 100):
        a, b = (llma.llma_attend_paged_mx(c, q[:m], i32([pages]), i32([200]), i32([0, m]), m, 0.09, torch.empty_like(q[:m])) for pages in (far, near))
        assert torch.equal(a, b) and a.float().abs().max() > 0.01
    rows = [[torch.empty((200, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    for pages, (k, v) in zip((far, near), rows):
        llma.llma_read_paged_mx(c, i32([pages]), None, i32([0, 200]), k, v)
    assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
    assert (rows[0][0].float() - x[:, 0].float()).abs().max() <= 1.0 and (rows[0][1].float() - x[:, 1].float()).abs().max() <= 1.0       # (half the largest step, 2, at scale 1)


# ------------------------------------------------------------------------------------------------ all of them together
def test_a_step_of_all_of_them_together_captured_and_replayed(llma):
    """map, append, attend, a look at the logits' log probabilities and the cache's rows, as a serving loop runs them, eagerly and as one graph replayed over growing sequences"""
    B, H, heads, D, m, blocks, V = 5, 2, 6, 64, 4, 6, 999
    rng = np.random.default_rng(81)
    rows = i32([m] * B)

    def state():
        pages = llma.PageTable.empty(B, blocks, B * blocks)
        cache = random_cache(llma, B * blocks, H, D, 9)
        bufs = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (B + 1, B, B * m, B * m, 1)]
        f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
        b16, i = torch.bfloat16, torch.int32
        return {"pages": pages, "cache": cache, "bufs": bufs, "lens": i32([0] * B), "x": f(B * m, heads + 2 * H, D, dt=b16), "out": f(B * m, heads, D, dt=b16),
                "w": f(heads * D, V, dt=b16), "logits": f(B * m, V, dt=b16), "tokens": f(B * m, dt=i), "logprob": f(B * m), "rank": f(B * m, dt=i), "entropy": f(B * m),
                "top": f(B * m, 3, dt=i), "top_lp": f(B * m, 3), "k": f(B * m, H, D), "v": f(B * m, H, D)}

    def step(s):
        off, after, slot_map, pos, status = s["bufs"]
        llma.llma_map_pages(s["pages"], s["lens"], rows, off, after, slot_map, pos, status)
        llma.llma_append_paged_mx(s["cache"], s["x"][:, heads:heads + H], s["x"][:, heads + H:], slot_map)
        llma.llma_attend_paged_mx(s["cache"], s["x"][:, :heads], s["pages"].table, after, off, m, D ** -0.5, s["out"])
        torch.matmul(s["out"].reshape(B * m, -1), s["w"], out=s["logits"])
        llma.llma_token_logprobs(s["logits"], s["tokens"], s["logprob"], rank=s["rank"], entropy=s["entropy"], top_tokens=s["top"], top_logprobs=s["top_lp"])
        llma.llma_read_paged_mx(s["cache"], s["pages"].table, s["lens"], off, s["k"], s["v"])

    eager, replayed = state(), state()
    w = torch.tensor(rng.standard_normal(eager["w"].shape), dtype=torch.bfloat16, device="cuda")
    for s in (eager, replayed):
        s["w"].copy_(w)
    step(eager)                                                         # (what the product's library sets up comes before the capture)
    eager = state()
    eager["w"].copy_(w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step(replayed)
    lens = np.zeros(B, int)
    for it in range(10):
        x = torch.tensor(rng.standard_normal(eager["x"].shape), dtype=torch.bfloat16, device="cuda")
        tokens = i32(rng.integers(0, V, B * m))
        for s in (eager, replayed):
            s["x"].copy_(x)
            s["lens"].copy_(i32(lens))
            s["tokens"].copy_(tokens)
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert eager["bufs"][4].item() == 0
        for name in ("out", "k", "v", "logprob", "rank", "entropy", "top", "top_lp"):
            if name in ("out", "k", "v") or torch.equal(eager["logits"], replayed["logits"]):
                assert torch.equal(eager[name], replayed[name]), name
        for a, b in zip(eager["bufs"], replayed["bufs"]):
            assert torch.equal(a, b)
        kv, vv = cached(eager["cache"])
        off, table = np.arange(B + 1) * m, eager["pages"].table.cpu().numpy()
        want, size, big = oracle.attend(kv, vv, x[:, :heads].double().cpu().numpy(), table, range(B), lens + m, off, D ** -0.5, B * blocks)
        tol = size * (2 * (D + 4) * 2.0 ** -24 * big + 2.0 ** -11 + 2.0 ** -12)[..., None] + 2.0 ** -8 * np.abs(want) + 1e-30
        assert (np.abs(eager["out"].double().cpu().numpy() - want) <= tol).all()
        for name, x0, values in (("k", heads, kv), ("v", heads + H, vv)):
            assert np.array_equal(eager[name].double().cpu().numpy(), mx.read(values, table, range(B), lens, off, B * m, B * blocks, 0.0), equal_nan=True)
            assert np.array_equal(eager[name].double().cpu().numpy(), mx.values(*mx.encode(x[:, x0:x0 + H].double().cpu().numpy())))
        for i in (0, 7, B * m - 1):
            lp, rank, entropy, top, _ = mx.logprobs(eager["logits"][i].double().cpu().numpy(), int(tokens[i]), 1.0, 3)
            assert abs(eager["logprob"][i].item() - lp) <= 1e-5 * (1 + abs(lp)) and eager["rank"][i].item() == rank and eager["top"][i].tolist() == top
        lens = lens + rng.integers(1, m + 1, B)                          # the accepted rows stay
        lens[rng.integers(0, B)] = 0                                     # one sequence ends, another begins in its place
        lens = np.minimum(lens, blocks * PAGE - m)


def test_rows_read_go_into_a_context(llma):
    """a prefix out of pages becomes a slot's cache in planes (llma_kv_import), whose step sees what an import of the same values sees"""
    import synth
    cfg = synth.WORKLOADS["small"].model
    w = synth.make_weights(cfg, 3)
    n, H, D = 130, cfg.n_heads, cfg.head_dim
    P = 4
    rng = np.random.default_rng(4)
    dumps = []
    caches = []
    for layer in range(cfg.n_layers):
        c = llma.PagedMxCache(*(t.zero_() for t in (lambda e: (e.k, e.v, e.k_scale, e.v_scale))(llma.PagedMxCache.empty(P, H, D))))
        x = torch.tensor(rng.standard_normal((n, 2, H, D)), dtype=torch.float32, device="cuda")
        llma.llma_append_paged_mx(c, x[:, 0], x[:, 1], i32(range(n)))
        caches.append(c)
    for by_read in (True, False):
        ctx = llma.Context(cfg, w, max_seq=256, max_batch=1, max_k=4)
        dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
        for layer, c in enumerate(caches):
            if by_read:
                k, v = (torch.empty((H, n, D), dtype=dt, device="cuda") for _ in range(2))
                llma.llma_read_paged_mx(c, i32([[0, 1, 2, 3]]), None, i32([0, n]), k.transpose(0, 1), v.transpose(0, 1))
            else:
                k, v = (torch.tensor(a.swapaxes(0, 1).reshape(H, P * PAGE, D)[:, :n].copy()).to(dt).cuda() for a in cached(c))
            ctx.kv_import(0, layer, k, v, n)
        ctx.set_pending(5)
        ctx.enable_logits_dump(8)
        ctx.verify_step([1, 2, 3])
        dumps.append(ctx.logits(4).copy())
        ctx.close()
    assert np.array_equal(dumps[0], dumps[1])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("lens,rows,heads,kv,D", [
    ([5000], [70], 2, 1, 64), ([3000, 1, 0, 900], [130, 1, 0, 300], 4, 2, 128), ([64 * 9 + 1], [200], 40, 40, 64), ([2000, 1999, 40], [129, 65, 90], 3, 1, 128),
    ([150, 400], [70, 3], 300, 300, 64)])
def test_attend_blocks_of_rows_in_several_shares(llma, dtype, lens, rows, heads, kv, D):
    """row blocks cut between workgroups: in the middle of a page list, over several of them, next to empty sequences and short ones"""
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 91, n_slots=len(lens) + 2, spare_rows=1)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype)


@pytest.mark.parametrize("rows", [3, 100])
def test_attend_slots_that_do_not_exist(llma, rows):
    """sequences whose slot is none see nothing: zeros; the others are as without them"""
    c, q, table, slots, off = attend_case(llma, [200, 200, 200], [rows] * 3, 4, 2, 64, "bf16", 95)
    args = (i32([200, 200, 200]), i32(off), rows, 0.125)
    clean = llma.llma_attend_paged_mx(c, q, i32(table), *args, torch.empty_like(q), slots=i32(slots))
    for bad in (-1, 3, 2 ** 31 - 1, -2 ** 31):
        got = llma.llma_attend_paged_mx(c, q, i32(table), *args, torch.full_like(q, 7.0), slots=i32([slots[0], bad, slots[2]]))
        assert not got[rows:2 * rows].any()
        assert torch.equal(got[:rows], clean[:rows]) or (got[:rows].float() - clean[:rows].float()).abs().max() <= 2.0 ** -6 * clean.float().abs().max()      # (cut elsewhere)
        assert (got[2 * rows:].float() - clean[2 * rows:].float()).abs().max() <= 2.0 ** -6 * clean.float().abs().max()


def test_attend_more_blocks_of_rows_than_a_list_holds(llma):
    """thousands of row blocks: a workgroup each"""
    B = 700
    rng = np.random.default_rng(97)
    lens = [int(x) for x in rng.integers(1, 200, B)]
    rows = [int(min(n, r)) for n, r in zip(lens, rng.integers(1, 140, B))]
    rows[3], lens[3] = 390, 400
    c, q, table, slots, off = attend_case(llma, lens, rows, 2, 2, 64, "bf16", 98)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), "bf16")


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows", [3, 30, 50, 130])
@pytest.mark.parametrize("shift,spread", [(0, 34), (-40, 3), (30, 3), (-22, 6), (11, 2)])
def test_attend_scales_far_from_one(llma, dtype, rows, shift, spread):
    """caches whose scales fp16 does not hold, or not all of them: small and large values of K and V, with queries and outputs in their types' range"""
    c, q, table, slots, off = attend_case(llma, [300], [rows], 4, 4, 64, dtype, 101, spread=0)
    rng = np.random.default_rng(7)
    for s in (c.k_scale, c.v_scale):
        r = torch.tensor(rng.integers(-spread, 1, s.shape), device="cuda")
        by = shift if s is c.k_scale or dtype != "fp16" else max(min(shift, 8), -16)        # (fp16 outputs end at 65504, and lose bits below 2^-14)
        s.copy_(torch.where(s == 255, 255, s.int() + by + r).to(torch.uint8))
    check_attend(llma, c, q, table, slots, [300], off, rows, dtype, scale=2.0 ** -(shift + 3))


def test_attend_subnormal_queries(llma):
    """fp16 queries below its normal range"""
    for rows in (3, 30, 130):
        c, q, table, slots, off = attend_case(llma, [300], [rows], 4, 2, 64, "fp16", 103, q_size=4e-6)
        check_attend(llma, c, q, table, slots, [300], off, rows, "fp16", scale=3e4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompts_captured_and_replayed(llma, dtype):
    """prompts in pieces: write, attention in the form for many rows, rows back, log probabilities of all rows; one graph, replayed with other lengths and tables between eager work"""
    B, H, heads, D, m, blocks, V = 3, 2, 8, 128, 90, 9, 2600
    P, n = B * blocks, B * m
    rng = np.random.default_rng(91)
    new = lambda *s, dt=DT[dtype]: torch.zeros(s, dtype=dt, device="cuda")
    at = {"table": i32(np.zeros((B, blocks))), "lens": i32([m] * B), "first": i32([0] * B), "off": i32([0, m, 2 * m, 3 * m]), "slots": i32([-1] * n), "tokens": i32([0] * n),
          "x": new(n, heads + 2 * H, D), "logits": new(n, V)}
    ws = torch.empty(llma.llma_attend_paged_mx_workspace(B, blocks, heads, H, D, m), dtype=torch.uint8, device="cuda")

    def state():
        return {"c": random_cache(llma, P, H, D, 7, nans=False), "out": new(n, heads, D), "k": new(n, H, D), "v": new(n, H, D), "lp": new(n, dt=torch.float32), "rank": new(n, dt=torch.int32),
                "top": new(n, 30, dt=torch.int32), "top_lp": new(n, 30, dt=torch.float32)}

    def step(s, work):
        llma.llma_append_paged_mx(s["c"], at["x"][:, heads:heads + H], at["x"][:, heads + H:], at["slots"])
        llma.llma_attend_paged_mx(s["c"], at["x"][:, :heads], at["table"], at["lens"], at["off"], m, D ** -0.5, s["out"], workspace=work)
        llma.llma_read_paged_mx(s["c"], at["table"], at["first"], at["off"], s["k"], s["v"])
        llma.llma_token_logprobs(at["logits"], at["tokens"], s["lp"], rank=s["rank"], top_tokens=s["top"], top_logprobs=s["top_lp"])

    eager, replayed = state(), state()
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=st):
        step(replayed, ws)
    for it in range(6):
        rows = rng.integers(0 if it else m, m + 1, B)
        lens = rows + rng.integers(0, blocks * PAGE - m, B)
        off = np.concatenate([[0], np.cumsum(rows)])
        table = rng.permutation(P).reshape(B, blocks)
        slots = np.full(n, -1)
        for b in range(B):
            pos = lens[b] - rows[b] + np.arange(rows[b])
            slots[off[b]:off[b + 1]] = table[b, pos // PAGE] * PAGE + pos % PAGE
        for name, value in (("table", table), ("lens", lens), ("first", lens - rows), ("off", off), ("slots", slots), ("tokens", rng.integers(0, V, n))):
            at[name].copy_(i32(value))
        for name in ("x", "logits"):
            at[name].copy_(torch.tensor(rng.standard_normal(at[name].shape), dtype=torch.float32))
        for o in (eager["out"], replayed["out"]):
            o.fill_(7.0)
        step(eager, None)
        graph.replay()
        torch.cuda.synchronize()
        for name in eager:
            if name != "c":
                assert torch.equal(eager[name], replayed[name]), (it, name)
        for a in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(eager["c"], a), getattr(replayed["c"], a))
        used = off[-1]
        assert np.array_equal(eager["k"][:used].float().cpu().numpy(), mx.values(*mx.encode(at["x"][:used, heads:heads + H].double().cpu().numpy())).astype(np.float32))
        keep = eager["out"].clone()
        # These scores lie so far apart that the largest probability's V, where its code is 0, leaves features to probabilities of 1e-10.  bf16 rows' are held in fp16, the largest of a row and
        # part of the pages as 2^7 or more: below fp16's normal range each is off by up to half a step, 2^-25, and so by up to 2^-32 of the largest, which is 1 at most.  2^-32 sum |v| in all
        # (twice, for the rounding of the sum that divides is of that size too, times an output of at most the largest |v|).
        _, vv = cached(eager["c"])
        besides = np.zeros((used, heads, D))
        for b in range(B):
            pos = np.arange(lens[b])
            v = np.abs(vv[table[b, pos // PAGE], :, pos % PAGE])
            besides[off[b]:off[b + 1]] = 2.0 ** -32 * (v.sum(0) + lens[b] * v.max(0, initial=0)).repeat(heads // H, 0)
        check_attend(llma, eager["c"], at["x"][:, :heads], table, range(B), lens, off, m, dtype, out=eager["out"], besides=besides if dtype == "bf16" else None)
        assert torch.equal(keep, eager["out"])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("lens,rows", [([130], [130]), ([300, 64], [70, 64])])
@pytest.mark.parametrize("rising", [True, False])
def test_attend_values_of_very_different_sizes_in_a_page(llma, dtype, lens, rows, rising):
    """scales of V that rise or fall by 2^31 inside each page: rows that see only its small ones have them exactly"""
    c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, 128, dtype, 111, q_size=0.2)
    step = torch.arange(PAGE, device="cuda").int() // 2
    by = (step if rising else 31 - step) - 20
    c.v_scale.copy_(torch.where(c.v_scale == 255, 255, c.v_scale.int() + by).to(torch.uint8))
    if dtype == "fp16":                                                 # (whose outputs end at 65504)
        c.v_scale.copy_(torch.where(c.v_scale == 255, 255, (c.v_scale.int() - 4)).to(torch.uint8))
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows", [[3, 5], [100, 41]])
@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-30])
def test_attend_scales_of_the_scores(llma, dtype, rows, scale):
    """all positions alike, the smallest product first"""
    lens = [170, 64]
    c, q, table, slots, off = attend_case(llma, lens, rows, 4, 2, 128, dtype, 121, q_size=1.0)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype, scale=scale)


def test_attend_infinite_queries_and_values(llma):
    """infinite scores, whose differences are no numbers, and NaN stay in their row and head"""
    for rows in ([4], [100]):
        lens = [150]
        c, q, table, slots, off = attend_case(llma, lens, rows, 2, 2, 128, "bf16", 131, q_size=1.0)
        out, bad = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
        args = (i32(table), i32(lens), i32(off), max(rows), 128 ** -0.5)
        llma.llma_attend_paged_mx(c, q, *args, out, slots=i32(slots))
        q[1, 0, 5] = float("inf")
        q[2, 1, 9] = float("nan")
        llma.llma_attend_paged_mx(c, q, *args, bad, slots=i32(slots))
        same = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
        same[1, 0] = same[2, 1] = False
        assert torch.equal(out[same], bad[same])
        assert bad[2, 1].isnan().all() and bad[1, 0].isnan().all()
