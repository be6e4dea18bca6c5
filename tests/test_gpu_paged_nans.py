"""NaN in V under the form of llma_attend_paged for many rows: every row that sees the position gets it, whether its page is seen whole or in part by the rows that
share the page's image; every other output is what it is without the NaN."""
import pytest
import torch

from test_gpu_paged import attend_case, i32, llma  # noqa: F401

pytestmark = pytest.mark.gpu


# lens, rows, heads, key heads, positions (of the second sequence): the block's first page, the page of a later wave's first row, one behind another block's first row
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,lens,rows,heads,kv,positions", [
    (64, [70, 300], [70, 300], 64, 64, [0, 63, 64, 127, 130, 255, 299]),       # fresh prompts, a head's own keys
    (128, [70, 300], [70, 300], 64, 64, [5, 70, 140]),
    (64, [40, 390], [40, 290], 64, 32, [101, 120, 130, 200, 389]),             # two query heads a key head, behind a cache of 100
    (128, [40, 390], [40, 290], 80, 16, [99, 100, 127, 160]),                  # five, blocks that begin inside a position's heads
])
def test_every_row_that_sees_it(llma, dtype, D, lens, rows, heads, kv, positions):  # noqa: F811
    c, q, table, slots, off = attend_case(llma, lens, rows, heads, kv, D, dtype, 17 + D + heads)
    group, block = heads // kv, 64 if dtype == "fp32" else 128
    assert max(rows) * group > 64 and min(len(rows) * -(-max(rows) * group // block), len(q) * group // block + len(rows)) * kv >= 160      # (the rule that picks the form)
    args = (i32(table), i32(lens), i32(off), max(rows), D ** -0.5)
    clean = llma.llma_attend_paged(c, q, *args, torch.empty_like(q), slots=i32(slots))
    assert clean.isfinite().all()
    for n, p in enumerate(positions):
        page, at, head, d = int(table[slots[1], p // 64]), p % 64, (5 * n + 3) % kv, (11 * n + 2) % D
        was = c.v[page, head, d, at].item()
        c.v[page, head, d, at] = 0xFF if n % 2 else 0x7F
        got = llma.llma_attend_paged(c, q, *args, torch.empty_like(q), slots=i32(slots))
        c.v[page, head, d, at] = was
        nan = torch.zeros_like(q, dtype=torch.bool)
        first = off[1] + max(0, p - (lens[1] - rows[1]))
        nan[first:, head * group:(head + 1) * group, d] = True
        assert torch.equal(got.isnan(), nan), (p, (got.isnan() != nan).nonzero()[:5].tolist())
        assert torch.equal(got[~nan], clean[~nan]), p
