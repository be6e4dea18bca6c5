"""Masks of the type's lowest value at an infinite temperature: they are above minus infinity, so llma_verify_sampled gives their tokens the others' weight."""
import numpy as np
import pytest
import torch

from test_gpu_sampled import DT, call, llma  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [50, 1003, 40000])
def test_sampled_tokens_have_equal_shares(llma, dtype, V):  # noqa: F811
    rng = np.random.default_rng(V)
    x = torch.tensor(5 * rng.standard_normal((2, V)), dtype=torch.float32).to(DT[dtype])
    x[0, ::2] = torch.finfo(DT[dtype]).min
    x[0, 1::7] = -INF
    x[0, 3] = float("nan")
    x[1] = torch.finfo(DT[dtype]).min
    x[1, V // 2] = 3.0
    x[1, 1::2] = torch.finfo(DT[dtype]).max                             # whose distance from the lowest is no number of the type
    B = 12
    live = [[v for v in range(V) if x[j, v] > -INF] for j in range(2)]
    logits = x.cuda().expand(B, 2, V).contiguous()
    n0, n1 = len(live[0]), len(live[1])
    temps = np.full(B, INF)
    at = rng.integers(0, n0 - 1, B)
    for draft in (live[0][n0 // 2], live[0][n0 // 2 + 1]):              # an ordinary one and one of lowest value, whichever comes first
        rest = [v for v in live[0] if v != draft]
        got = call(llma, logits, np.full((B, 1), draft), np.full((B, 1), 0.99 / n0), (at + 0.5) / n1, temperature=temps)
        assert (got[0] == 1).all() and got[1].tolist() == [live[1][a] for a in at]
        got = call(llma, logits, np.full((B, 1), draft), np.full((B, 1), 1.01 / n0), (at + 0.5) / (n0 - 1), temperature=temps)
        assert (got[0] == 0).all() and got[1].tolist() == [rest[a] for a in at]
        q = torch.zeros((B, 1, V), device="cuda")
        q[:, :, draft] = 1.0
        got = call(llma, logits, np.full((B, 1), draft), np.full((B, 1), 0.5), (at + 0.5) / (n0 - 1), probs=q, temperature=temps)
        assert (got[0] == 0).all() and got[1].tolist() == [rest[a] for a in at]
    # an infinite logit takes all, whatever the temperature
    logits[:, 0, 9] = INF
    got = call(llma, logits[:, :1], np.zeros((B, 0)), np.zeros((B, 0)), (at + 0.5) / n0, temperature=temps)
    assert (got[1] == 9).all()
