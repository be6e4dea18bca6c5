"""Masks of the type's lowest value at an infinite temperature: they are above minus infinity, so llma_token_logprobs gives their tokens the others' probability."""
import numpy as np
import pytest
import torch

from test_gpu_logprobs import DT, check, llma  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


def masked(V, dtype, seed):
    """half of the tokens at the type's lowest value, a seventh at minus infinity, some NaN; all but one at the lowest; large logits beside the lowest"""
    rng = np.random.default_rng(seed)
    x = torch.tensor(5 * rng.standard_normal((4, V)), dtype=torch.float32).to(DT[dtype])
    low = torch.finfo(DT[dtype]).min
    x[0, ::2] = low
    x[0, 1::7] = -INF
    x[0, 3] = float("nan")
    x[1] = low
    x[1, V // 2] = 3.0
    x[2, ::3] = -low                                                    # the largest there is
    x[2, 1::3] = low
    x[3, ::2] = -INF
    return x


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [7, 999, 32000, 50257])
def test_logprobs_are_alike(llma, dtype, V):  # noqa: F811
    x = masked(V, dtype, V).cuda()
    for tokens in ([0, 0, 0, 1], [4, V // 2, 1, V - 1], [1, 1, 2, 0]):
        got = check(llma, x, tokens, [INF] * 4, 5)
        assert abs(got["entropy"][1] - np.log(V)) < 1e-5 * np.log(V)
    # an infinite logit still takes all, with others of lowest value or ordinary ones beside it
    x[0, 5 % V] = x[1, 2] = x[2, 3] = INF
    check(llma, x, [5 % V, 0, 3, 1], [INF] * 4, 5)
