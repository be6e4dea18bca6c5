"""llma_map_pages without a slot map: tables, stack, offsets and lengths of a step with rows are those of a call with one."""
import numpy as np
import pytest
import torch

from test_gpu_paged import Pages, i32, llma  # noqa: F401

pytestmark = pytest.mark.gpu


def outputs(B, cap):
    return [torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (B + 1, B, cap, cap, 1)]


@pytest.mark.parametrize("B", [1, 5, 300, 1100])
@pytest.mark.parametrize("named", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_rows_without_a_map(llma, B, named, given):  # noqa: F811
    """None in place of the map, and a map of no entries; a second call on the grown lengths, a third that gives pages back"""
    rng = np.random.default_rng(B)
    n_slots, blocks = B + 3, 40
    a, b = (Pages(llma, n_slots, blocks, n_slots * blocks, np.random.default_rng(2)).dev for _ in range(2))
    slots = i32(rng.permutation(n_slots)[:B]) if named else None
    lens = rng.integers(0, 700, n_slots)
    for rows in (rng.integers(0, 500, B), rng.integers(1, 900, B), np.zeros(B, int)):
        cap = max(1, int(rows.sum()))
        want, got = outputs(B, cap), outputs(B, 0)
        llma.llma_map_pages(a, i32(lens), i32(rows), *want, slots=slots)
        llma.llma_map_pages(b, i32(lens), i32(rows), got[0], got[1], got[2] if given else None, got[3] if given else None, got[4], slots=slots)
        assert want[4].item() == 0 and got[4].item() == 0
        for i in (0, 1):
            assert torch.equal(want[i], got[i])
        assert got[0][-1].item() == rows.sum()
        n = a.n_free.item()
        assert b.n_free.item() == n and torch.equal(a.free_pages[:n], b.free_pages[:n])
        assert torch.equal(a.table, b.table) and torch.equal(a.owned, b.owned)


def test_a_map_of_one_entry_is_not_no_map(llma):  # noqa: F811
    """two rows where one has a place: refused, nothing changed"""
    pages = Pages(llma, 2, 4, 8, np.random.default_rng(3)).dev
    got = outputs(2, 1)
    llma.llma_map_pages(pages, i32([5, 60]), i32([1, 1]), *got)
    assert got[4].item() == llma.LLMA_E_RANGE and got[0].tolist() == [0, 0, 0] and got[2].item() == -1 and pages.n_free.item() == 8


@pytest.mark.parametrize("B", [64, 65, 128, 129, 1024, 1100])
def test_page_counts_past_32_bits(llma, B):  # noqa: F811
    """sequences that each want, or own, all of a table's width: their sums pass 2^31 and 2^32.  Missing pages are counted (2^31 - 1 at most), nothing is changed"""
    total = 130 << 25                                                    # entries of a table, 17 GB (never touched: no page is granted)
    blocks = min((1 << 25) - 1, total // B)
    free = 10
    pages = llma.PageTable(torch.empty((B, blocks), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"),
                           torch.arange(free, dtype=torch.int32, device="cuda"), i32([free]))
    for lens, rows in ((blocks * 64 - 5, 3), (0, blocks * 64), (blocks * 64, 0)):
        got = outputs(B, 0)
        llma.llma_map_pages(pages, i32([lens] * B), i32([rows] * B), got[0], got[1], None, None, got[4])
        missing, too_many = B * blocks - free, B * rows > 0x7fffffff
        assert got[4].item() == (llma.LLMA_E_RANGE if too_many else min(missing, 0x7fffffff))
        assert not got[0].any() and (got[1] == lens).all() and not pages.owned.any() and pages.n_free.item() == free
    pages.owned.fill_(blocks)                                            # more pages than there are
    got = outputs(B, 0)
    llma.llma_map_pages(pages, i32([0] * B), i32([1] * B), got[0], got[1], None, None, got[4])
    assert got[4].item() == llma.LLMA_E_INVAL and (pages.owned == blocks).all() and pages.n_free.item() == free
