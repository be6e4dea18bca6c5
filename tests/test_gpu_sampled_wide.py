"""llma_verify_sampled where a row has more than 256 of the ranges whose sums it keeps (above 524288 fp32 or 1048576 bf16 / fp16 tokens): random numbers spread over [0, 1)
against the plain numpy form in 64 bits."""
import numpy as np
import pytest
import torch

import paged_oracle as oracle
from test_gpu_sampled import DT, call, llma  # noqa: F401

pytestmark = pytest.mark.gpu


def case(V, dtype, seed, flat):
    rng = np.random.default_rng(seed)
    x = torch.tensor(rng.standard_normal((2, V), dtype=np.float32) * np.float32(0.0 if flat else 1.5)).to(DT[dtype])
    return x, rng


@pytest.mark.parametrize("V,dtype", [(600001, "fp32"), (1100003, "bf16"), (1500001, "bf16"), (2200000, "fp16"), (1600000, "fp32")])
@pytest.mark.parametrize("flat", [False, True])
def test_tokens_of_wide_rows(llma, V, dtype, flat):  # noqa: F811
    """16 sequences over the same two rows: all drafts accepted, then drawn from p; the copied draft rejected and drawn from the rest"""
    rows, rng = case(V, dtype, V, flat)
    B = 16
    logits = rows.cuda().expand(B, 2, V).contiguous()
    us = ((np.arange(B) + rng.random(B)) / B).astype(np.float32)
    us[0], us[-1] = 0.0, np.float32(1) - np.float32(2.0 ** -24)
    drafts = rng.integers(0, V, (B, 1))
    x = rows.double().numpy()
    for ua in (np.zeros((B, 1), np.float32), np.full((B, 1), 0.99, np.float32)):
        got = call(llma, logits, drafts, ua, us)
        for b in range(B):
            n, token, emitted, near = oracle.verify(x, drafts[b], 1, None, 1.0, ua[b], us[b])
            assert near > 1e-13 and n == (1 if ua[b, 0] == 0 else 0)
            assert (got[0][b], got[1][b]) == (n, token), (b, float(us[b]))


@pytest.mark.parametrize("V,dtype", [(600001, "fp32"), (1100003, "bf16")])
@pytest.mark.parametrize("cover", ["none", "half", "all"])
def test_tokens_left_by_draft_probabilities(llma, V, dtype, cover):  # noqa: F811
    """rejected drafts: drawn from max(p - q, 0), where q leaves nothing from p; q that covers the first half moves the target into later ranges"""
    rows, rng = case(V, dtype, V + 1, False)
    B = 8
    p = torch.softmax(rows[0].double(), 0)
    q = {"none": torch.roll(p, 1000), "half": torch.where(torch.arange(V) < V // 2, p * 1.5, p * 0.1), "all": p * 2}[cover].float()
    logits = rows.cuda().expand(B, 2, V).contiguous()
    us = ((np.arange(B) + rng.random(B)) / B).astype(np.float32)
    drafts = rng.integers(0, V, (B, 1))
    ua = np.full((B, 1), 0.999999, np.float32)
    q[torch.tensor(drafts[:, 0])] = (3 * p[torch.tensor(drafts[:, 0])]).float()          # (rejected)
    got = call(llma, logits, drafts, ua, us, probs=q.cuda().expand(B, 1, V).contiguous())
    x, pr = rows.double().numpy(), q.numpy()[None]
    for b in range(B):
        n, token, emitted, near = oracle.verify(x, drafts[b], 1, pr, 1.0, ua[b], us[b])
        assert near > 1e-13 and n == 0
        assert (got[0][b], got[1][b]) == (n, token), (b, float(us[b]))


@pytest.mark.parametrize("V,dtype", [(3000001, "fp32"), (1 << 23, "bf16")])
def test_tests_next_to_their_border(llma, V, dtype):  # noqa: F811
    """copied drafts with random numbers from 1e-7 to 1e-3 of their probability below and above it: sums over hundreds of chunks, all alike, do not tell the nearest"""
    rows = torch.full((2, V), -1.2345)
    rows[:, 77] = 6.0
    rows = rows.to(DT[dtype])
    x = rows.double().numpy()
    w = np.exp(x[0] - x[0].max())
    B = 24
    ua = np.zeros((B, 1), np.float32)
    draft = 77
    p = w[draft] / w.sum()
    for b in range(B):
        off = 10.0 ** (-7 + b // 2 * 4 / 11)
        ua[b, 0] = np.float32(p * (1 + (off if b % 2 else -off)))
    logits = rows.cuda().expand(B, 2, V).contiguous()
    got = call(llma, logits, np.full((B, 1), draft), ua, np.full(B, 0.3, np.float32))
    assert got[0].tolist() == [int(float(u) < p) for u in ua[:, 0]] and 0 < got[0].sum() < B
