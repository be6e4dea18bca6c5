"""llma_verify_sampled at temperatures that leave nothing of the logits: every token with a logit above minus infinity has the same weight, masked ones none."""
import numpy as np
import pytest
import torch

from test_gpu_sampled import DT, call, llma  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T", [1e30, 1e38, 3e38, float("inf")])
@pytest.mark.parametrize("V", [50, 1003, 40000])
def test_uniform_over_what_can_be(llma, dtype, T, V):  # noqa: F811
    """tokens at random numbers in the middles of equal shares; drafts accepted below 1 / n and not above, a masked one never; draft probabilities"""
    rng = np.random.default_rng(V)
    x = torch.tensor(rng.standard_normal((2, V)) * 5.0).to(DT[dtype])
    x[:, ::3] = -float("inf")
    x[0, 4] = float("nan")
    live = [[v for v in range(V) if v % 3 and (j or v != 4)] for j in range(2)]
    B = 12
    logits = x.cuda().expand(B, 2, V).contiguous()
    n0, n1 = len(live[0]), len(live[1])
    draft = live[0][n0 // 2]
    rest = [v for v in live[0] if v != draft]
    at = rng.integers(0, n0 - 1, B)
    temps = np.full(B, T)
    # accepted: from the second row, whose shares are 1 / n1
    got = call(llma, logits, np.full((B, 1), draft), np.full((B, 1), 0.99 / n0), (at + 0.5) / n1, temperature=temps)
    assert (got[0] == 1).all() and got[1].tolist() == [live[1][a] for a in at]
    # rejected: from the first row without the draft
    got = call(llma, logits, np.full((B, 1), draft), np.full((B, 1), 1.01 / n0), (at + 0.5) / (n0 - 1), temperature=temps)
    assert (got[0] == 0).all() and got[1].tolist() == [rest[a] for a in at]
    # a masked draft, and one that is NaN: never, and all of the row is left
    for token in (3, 4):
        got = call(llma, logits, np.full((B, 1), token), np.zeros((B, 1)), (at + 0.5) / n0, temperature=temps)
        assert (got[0] == 0).all() and got[1].tolist() == [live[0][a] for a in at]
    # draft probabilities of one token: max(p - q, 0) is p elsewhere
    q = torch.zeros((B, 1, V), device="cuda")
    q[:, :, draft] = 1.0
    got = call(llma, logits, np.full((B, 1), draft), np.full((B, 1), 0.5), (at + 0.5) / (n0 - 1), probs=q, temperature=temps)
    assert (got[0] == 0).all() and got[1].tolist() == [rest[a] for a in at]


def test_nothing_to_choose_from(llma):  # noqa: F811
    logits = torch.full((2, 1, 70), -float("inf"), device="cuda")
    logits[1, 0, 9] = 2.0
    got = call(llma, logits, np.zeros((2, 0)), np.zeros((2, 0)), np.array([0.5, 0.5]), temperature=np.full(2, float("inf")))
    assert got[1].tolist() == [-1, 9]
