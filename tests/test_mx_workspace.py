"""The workspace of attention over 4-bit pages: what is asked for some number of sequences does for fewer, also where the number decides which kernel a call takes (no GPU needed)."""
import pytest

import paper_2304_04487_amd as llma


def most_sequences(blocks, rows, heads):
    """that a call with such tables takes"""
    return min(llma.LLMA_PAGED_MAX_SEQS, (2 ** 31 - 1) // 64 // blocks)


@pytest.mark.parametrize("blocks", [3, 100, 128, 500, 1024, 8000])
@pytest.mark.parametrize("heads,kv,dh", [(32, 8, 128), (64, 8, 128), (128, 128, 128), (8, 8, 64), (64, 8, 64), (256, 256, 128), (32, 1, 64), (600, 300, 128), (1024, 1024, 64)])
@pytest.mark.parametrize("rows", [1, 9, 33, 65, 300, 2000, 8192, 65536])
def test_more_sequences_never_ask_for_less(blocks, heads, kv, dh, rows):
    top = most_sequences(blocks, rows, heads)
    counts = sorted({n for n in (1, 2, 3, 5, 7, 16, 30, 64, 128, 200, 500, 511, 512, 700, 1000, 1023, 1024, 1025, 1500, 2000, 2047, 2048, 2049, 3000, 4000, 4095, 4096, top) if n <= top})
    sizes = [llma.llma_attend_paged_mx_workspace(n, blocks, heads, kv, dh, rows) for n in counts]
    assert sizes == sorted(sizes), list(zip(counts, sizes))
    assert sizes[-1] < 70 << 20
