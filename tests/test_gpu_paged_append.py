"""llma_append_paged where a page's scale grows: codes before the run rounded again, the run's own and those behind it as the definition has them, bit for bit; runs of
steps and, with several waves a page, of prompts."""
import numpy as np
import pytest
import torch

import paged_oracle as oracle
from test_gpu_paged import DT, PAGE, cache_values, i32, llma, random_cache  # noqa: F401

pytestmark = pytest.mark.gpu


def check(llma, c, x, slot_map):  # noqa: F811
    want = cache_values(c)
    exact = x.double().cpu().numpy()
    oracle.append(want[0], want[2], exact[:, 0], slot_map)
    oracle.append(want[1], want[3], exact[:, 1], slot_map)
    before = cache_values(c)
    llma.llma_append_paged(c, x[:, 0], x[:, 1], i32(slot_map))
    got = cache_values(c)
    for g, w, part in zip(got, want, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(g, w, equal_nan=True), part
    return got[2] > before[2]                              # the pages whose scale grew


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", list(DT))
def test_every_offset_of_a_step(llma, D, dtype):  # noqa: F811
    """a run of three rows at each position of a page that leaves room for it, values of 1 to 1000 over pages whose scales are 2^-9 to 2^3"""
    rng = np.random.default_rng(D)
    c = random_cache(llma, 62, 2, D, 13)
    slot_map = [p * PAGE + p + i for p in range(62) for i in range(3)]
    x = torch.tensor(rng.standard_normal((len(slot_map), 2, 2, D)) * 10.0 ** rng.integers(0, 4, (len(slot_map), 2, 2, 1))).to(DT[dtype]).cuda()
    grew = check(llma, c, x, slot_map)
    assert grew.any() and not grew.all()


@pytest.mark.parametrize("D,rows", [(128, 640), (64, 1200)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompts_that_begin_inside_a_page(llma, D, rows, dtype):  # noqa: F811
    """several waves a page: two prompts that begin at positions 61 and 18 of pages with other rows in them"""
    rng = np.random.default_rng(D + rows)
    H, P = 32, rows // PAGE + 5
    assert (rows + 63) // 64 * 2 * H * (4 if D == 128 else 2) >= 2048        # (the rule that picks the form)
    c = random_cache(llma, P, H, D, 17)
    pages = rng.permutation(P)
    cut = rows // 3
    slot_map, at = [], 0
    for off, n in ((61, cut), (18, rows - cut)):
        slot_map += [int(pages[at + (off + i) // PAGE]) * PAGE + (off + i) % PAGE for i in range(n)]
        at += (off + n + PAGE - 1) // PAGE
    assert at <= P
    x = torch.tensor(rng.standard_normal((rows, 2, H, D)) * 300).to(DT[dtype]).cuda()
    assert check(llma, c, x, slot_map).any()


@pytest.mark.parametrize("D", [64, 128])
def test_short_and_long_runs_together(llma, D):  # noqa: F811
    """steps of many sequences: runs of 1 to 64 rows at any offset, several in a window of 64 rows, some over its end"""
    rng = np.random.default_rng(D)
    H, P = 32, 110
    c = random_cache(llma, P, H, D, 19)
    slot_map = []
    for i, page in enumerate(rng.permutation(P)[:100]):
        off = int(rng.integers(0, PAGE)) if i % 3 else 0
        n = int(min(PAGE - off, rng.integers(1, 6) if i % 4 else rng.integers(14, 65)))
        slot_map += [int(page) * PAGE + off + j for j in range(n)] + [-1] * (i % 5 == 0)
    slot_map += [-1] * max(0, 1100 - len(slot_map))        # (the form with several waves a page)
    x = torch.tensor(rng.standard_normal((len(slot_map), 2, H, D)) * 10.0 ** rng.integers(0, 4, (len(slot_map), 2, H, 1))).bfloat16().cuda()
    assert check(llma, c, x, slot_map).any()
