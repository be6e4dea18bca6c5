"""Calls at the limits that llma.h names and between the shapes of the other tests: the most sequences, slots, heads and rows; rows of q that lie on each other; max_rows and tables far larger than
what is there; several calls at once on streams of their own.  All against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import paged_oracle as oracle
from test_gpu_paged import DT, PAGE, Pages, attend_case, cache_values, check_attend, i32, llma, random_cache  # noqa: F401
from test_gpu_sampled import call, check, inputs

pytestmark = pytest.mark.gpu


def test_map_65536_slots(llma):  # noqa: F811
    """all of them in one call, in a shuffled order; a second that gives half back and takes others"""
    rng = np.random.default_rng(1)
    S = 65536
    pages = Pages(llma, S, 2, S + 1000, rng)
    lens = [0] * S
    for turn in range(2):
        slots = [int(s) for s in rng.permutation(S)]
        rows = [int(r) for r in rng.integers(0, 3, S)] if turn else [1] * S
        if turn:
            for s in slots[::2]:
                lens[s] = 0
        got, want = pages.step(slots, lens, rows, sum(rows) + 7)
        pages.check(got, want)
        for s, r in zip(slots, rows):
            lens[s] += r


@pytest.mark.parametrize("D,heads,kv", [(64, 71, 1), (128, 200, 1), (64, 1024, 1024), (64, 2048, 1024)])
def test_head_layouts(llma, D, heads, kv):  # noqa: F811
    lens, rows = [70, 3], [2, 1]
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, "bf16", 5)
    check_attend(llma, c, q, table, slots, lens, off, 2, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_4096_sequences(llma, dtype):  # noqa: F811
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, 90, 4096)]
    rows = [int(rng.integers(0, 2)) for _ in lens]
    c, q, table, slots, off = attend_case(llma, lens, rows, 2, 1, 64, dtype, 6, spare_rows=2)
    for t in (table, np.concatenate([table, np.full((len(table), 50), -1)], 1)):         # whole, cut
        check_attend(llma, c, q, t, slots, lens, off, 1, dtype)


@pytest.mark.parametrize("max_rows", [9, 200, 3000])
def test_max_rows_far_above_the_rows(llma, max_rows):  # noqa: F811
    for heads, kv, lens, rows in ((4, 2, [300, 40, 0, 1000], [9, 1, 0, 3]), (64, 64, [400, 90], [9, 2])):
        c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, 64, "fp16", 7, spare_rows=1)
        check_attend(llma, c, q, table, slots, lens, off, max_rows, "fp16")


def test_rows_of_q_on_top_of_each_other_and_rows_before_the_first_sequence(llma):  # noqa: F811
    lens, rows = [150, 90], [9, 4]
    c, q, table, slots, off = attend_case(llma, lens, rows, 8, 2, 64, "bf16", 8)
    for shared in (q[:1].expand(13, 8, 64), q[:, :1].expand(13, 8, 64), q[:1, :1].expand(13, 8, 64)):
        want = llma.llma_attend_paged(c, shared.contiguous(), i32(table), i32(lens), i32(off), 9, 0.125, torch.zeros_like(q), slots=i32(slots))
        got = llma.llma_attend_paged(c, shared, i32(table), i32(lens), i32(off), 9, 0.125, torch.zeros_like(q), slots=i32(slots))
        assert torch.equal(got, want)
    moved = torch.cat([torch.full_like(q[:3], 9.0), q])
    out = torch.full_like(moved, 7.0)
    llma.llma_attend_paged(c, moved, i32(table), i32(lens), i32(np.asarray(off) + 3), 9, 0.125, out, slots=i32(slots))
    want = llma.llma_attend_paged(c, q, i32(table), i32(lens), i32(off), 9, 0.125, torch.zeros_like(q), slots=i32(slots))
    assert (out[:3] == 7.0).all() and torch.equal(out[3:], want)


def test_append_1024_heads(llma):  # noqa: F811
    H, D = 1024, 64
    rng = np.random.default_rng(9)
    c = random_cache(llma, 3, H, D, 3)
    slot_map = [2 * PAGE + 60 + i for i in range(4)] + [i for i in range(9)]
    x = torch.tensor(rng.standard_normal((13, 2, H, D)), dtype=torch.bfloat16).cuda()
    want = cache_values(c)
    oracle.append(want[0], want[2], x[:, 0].double().cpu().numpy(), slot_map)
    oracle.append(want[1], want[3], x[:, 1].double().cpu().numpy(), slot_map)
    llma.llma_append_paged(c, x[:, 0], x[:, 1], i32(slot_map))
    for g, w in zip(cache_values(c), want):
        assert np.array_equal(g, w, equal_nan=True)


@pytest.mark.parametrize("B,k,V", [(1 << 22, 0, 3), (1 << 16, 63, 2), (3, 63, 1), (9000, 2, 5)])
def test_verify_many_rows(llma, B, k, V):  # noqa: F811
    """the most rows: every sequence one of a hundred, of which the plain form knows the answer"""
    n = min(B, 100)
    logits, drafts, ua, us, _ = inputs(n, k, V, "fp32", 4)
    rng = np.random.default_rng(B)
    which = rng.integers(0, n, B)
    want = check(llma, logits, drafts, ua, us)
    idx = torch.tensor(which, device="cuda")
    got = call(llma, logits[idx], drafts[which], ua[which], us[which])
    for g, w in zip(got, want):
        assert np.array_equal(g, w[which])


def test_several_calls_at_once(llma):  # noqa: F811
    """four streams, each with its own attention, verification and write over and over, workspaces of the caller's and of the call's: all as by themselves"""
    cases, wants = [], []
    for i in range(4):
        lens, rows = [700 + 50 * i, 90, 2000], [9, 1, 5]
        c, q, table, slots, off = attend_case(llma, lens, rows, 16, 8, 64, ["bf16", "fp16", "fp32", "bf16"][i], 50 + i)
        logits, drafts, ua, us, _ = inputs(3, 4, 5000 + i, "bf16", 60 + i)
        ver = (logits, i32(drafts), torch.tensor(ua, device="cuda"), torch.tensor(us, device="cuda"))
        att = (c, q, i32(table), i32(lens), i32(off), 9, 0.125)
        wants.append((llma.llma_attend_paged(*att, torch.zeros_like(q), slots=i32(slots)).clone(), call(llma, logits, drafts, ua, us)))
        cases.append((att, i32(slots), ver, torch.cuda.Stream(), torch.empty(llma.llma_attend_paged_workspace(3, table.shape[1], 16, 8, 64, 9), dtype=torch.uint8, device="cuda"),
                      torch.zeros_like(q), [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((3,), (3,), (3, 5))]))
    torch.cuda.synchronize()
    for turn in range(20):
        for att, slots, ver, st, ws, out, res in cases:
            llma.llma_attend_paged(*att, out, slots=slots, stream=st, workspace=ws if turn % 2 else None)
            llma.llma_verify_sampled(*ver, *res, stream=st)
    torch.cuda.synchronize()
    for (att, slots, ver, st, ws, out, res), (a, v) in zip(cases, wants):
        assert torch.equal(out, a)
        for g, w in zip(res, v):
            assert np.array_equal(g.cpu().numpy(), w)
