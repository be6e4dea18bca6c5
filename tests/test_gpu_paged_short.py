"""llma_attend_paged over short sequences, which it takes whole or cut into shares by the width of the table: the same sequences under a table as wide as they
need and under a wider one, both against the plain numpy form in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_paged import attend_case, check_attend, i32, llma  # noqa: F401

pytestmark = pytest.mark.gpu


def widen(table, blocks, rng):
    """more columns, of numbers that are no sequence's pages or no pages at all"""
    return np.concatenate([table, rng.integers(-5, 99, (len(table), blocks - table.shape[1]))], axis=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,heads,kv,lens,rows", [
    (64, 8, 8, [1, 64, 0, 130, 2, 257], [1, 1, 2, 1, 0, 6]),
    (128, 4, 1, [5, 900, 64, 70, 1500, 1], [3, 9, 9, 1, 5, 1]),
    (128, 32, 32, [700], [9]),
    (64, 12, 2, [383, 2, 129], [33, 2, 40]),
    (128, 40, 8, [640, 65, 1, 300] * 5, [9, 1, 1, 13] * 5),
    (64, 2, 1, [int(x) for x in np.exp(np.linspace(0, 6.9, 300))], [1] * 300),         # more sequences than a workgroup's threads
])
def test_whole_and_cut(llma, dtype, D, heads, kv, lens, rows):  # noqa: F811
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 71 + D + heads, n_slots=len(lens) + 3, spare_rows=2)
    rng = np.random.default_rng(1)
    outs = []
    for blocks in (table.shape[1], 41, 64):                                            # (tables of more than 40 columns: cut)
        wide = widen(table, blocks, rng) if blocks > table.shape[1] else table
        outs.append(check_attend(llma, c, q, wide, slots, lens, off, max(rows), dtype))
    # where the pages are cut depends on their number alone, not on the table's width
    assert torch.equal(outs[1], outs[2])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_empty_whole_sequences(llma, dtype):  # noqa: F811
    """no positions, no rows, pages that do not exist: zeros where nothing is seen, other rows as they were"""
    lens, rows = [0, 70, 3, 0, 128], [2, 0, 3, 0, 1]
    c, q, table, slots, off = attend_case(llma, lens, rows, 8, 4, 64, dtype, 75, spare_rows=3)
    table[slots[2], 0] = len(c.k)                          # no such page
    for blocks in (table.shape[1], 50):
        t = widen(table, blocks, np.random.default_rng(2)) if blocks > table.shape[1] else table
        out = torch.full_like(q, 7.0)
        llma.llma_attend_paged(c, q, i32(t), i32(lens), i32(off), 3, 0.125, out, slots=i32(slots))
        assert not out[:5].any() and (out[6:] == 7.0).all() and out[5].isfinite().all() and out[5].any()


def test_a_workspace_for_more_sequences_does_for_fewer(llma):  # noqa: F811
    for heads, kv, D, rows in ((32, 32, 128, 9), (8, 8, 64, 1), (32, 8, 128, 5), (32, 8, 128, 20)):
        for blocks in (1, 9, 16, 32, 40, 41, 64):
            need = [llma.llma_attend_paged_workspace(n, blocks, heads, kv, D, rows) for n in range(1, 70)]
            assert need == sorted(need)
