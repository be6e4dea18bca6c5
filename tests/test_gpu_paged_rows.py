"""llma_attend_paged's form for many rows (more than 64 a key head, and at least 160 row blocks in the call) against the plain numpy form in 64 bits: row blocks and waves
that end inside a sequence, pages that end inside a row block, rows that see nothing, NaN that only later rows see, all row types."""
import numpy as np
import pytest
import torch

from test_gpu_paged import attend_case, check_attend, i32, llma  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,heads,kv,lens,rows", [
    (128, 32, 32, [70, 130, 64, 200, 81, 66], [70, 65, 64, 1, 80, 66]),
    (64, 32, 32, [70, 130, 64, 200, 81, 66], [70, 65, 64, 1, 80, 66]),
    (128, 64, 64, [300], [257]),
    (64, 64, 8, [90, 20, 700, 128], [90, 20, 33, 128]),
    (128, 48, 16, [129, 63, 190], [129, 63, 150]),
    (64, 42, 42, [4200], [390]),                           # more than 64 pages
])
def test_rows(llma, dtype, D, heads, kv, lens, rows):  # noqa: F811
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 91 + D + heads, n_slots=len(lens) + 2, spare_rows=2)
    group, block = heads // kv, 64 if dtype == "fp32" else 128
    blocks = min(len(rows) * -(-max(rows) * group // block), len(q) * group // block + len(rows)) * kv
    assert max(rows) * group > 64 and blocks >= 160        # (the rule that picks the form)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype)
    check_attend(llma, c, q, table, slots, lens, off, max(rows), dtype, scale=-0.2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_see_nothing(llma, dtype):  # noqa: F811
    lens, rows = [5, 0, 130, 70], [90, 70, 66, 70]
    c, q, table, slots, off = attend_case(llma, lens, rows, 64, 64, 64, dtype, 95, q_size=1.0)
    table[slots[2], 1] = len(c.k) + 3                      # no such page
    out = check_attend(llma, c, q, table, slots, lens, off, 90, dtype, scale=0.0)
    assert not out[:85].any() and not out[90:160].any() and out[85].any()


def test_nan_stays_in_rows_that_see_it(llma):  # noqa: F811
    lens, rows = [70, 200], [70, 80]
    for which in ("v", "k", "q"):
        c, q, table, slots, off = attend_case(llma, lens, rows, 96, 96, 64, "bf16", 97)
        args = (i32(table), i32(lens), i32(off), 80, 0.125)
        clean = llma.llma_attend_paged(c, q, *args, torch.empty_like(q), slots=i32(slots))
        page = int(table[slots[1], 2])                     # positions 128 .. 191 of the second sequence, whose rows are 120 .. 199
        if which == "v":
            c.v[page, 7, 5, 2] = 0x7F
        elif which == "k":
            c.k[page, 7, 2, 5] = 0xFF
        else:
            q[100, 7, 9] = float("nan")
        got = llma.llma_attend_paged(c, q, *args, torch.empty_like(q), slots=i32(slots))
        nan = torch.zeros_like(q, dtype=torch.bool)
        if which == "v":
            nan[70 + 10:, 7, 5] = True
        elif which == "k":
            nan[70 + 10:, 7, :] = True
        else:
            nan[100, 7, :] = True
        assert torch.equal(got.isnan(), nan), which
        assert torch.equal(got[~nan], clean[~nan]), which


def test_a_prompts_rows_are_those_of_its_steps(llma):  # noqa: F811
    """the two forms against each other: a row's output in a call of many rows and in a call of its own, to the sum of both forms' tolerances (four steps
    of bf16: one probability rounding and one output rounding each, on outputs that are averages of positive numbers)"""
    lens, rows = [700], [640]
    c, q, table, slots, off = attend_case(llma, lens, rows, 40, 40, 128, "bf16", 99)
    c.v &= 0x7F                                            # (signs off: outputs are as large as what they average)
    many = llma.llma_attend_paged(c, q, i32(table), i32(lens), i32(off), 640, 0.1, torch.empty_like(q), slots=i32(slots)).float()
    for j in (0, 1, 63, 64, 127, 128, 500, 639):
        one = llma.llma_attend_paged(c, q[j:j + 1], i32(table), i32([60 + j + 1]), i32([0, 1]), 1, 0.1, torch.empty_like(q[:1]), slots=i32(slots)).float()
        assert ((many[j] - one[0]).abs() <= 4 * 2.0 ** -8 * one[0].abs() + 1e-6).all(), j
