"""llma_token_logprobs at temperatures near zero over rows whose largest logit is zero, as rows from which their maximum was taken, or certain tokens' log probabilities, have it."""
import numpy as np
import pytest
import torch

import mx_oracle as mx
from test_gpu_logprobs import DT, llma, near, run  # noqa: F401

pytestmark = pytest.mark.gpu
FLT_MAX = float(np.finfo(np.float32).max)


def rows_at_zero(V):
    """max-subtracted; all alike; certain; certain, the rest the type's lowest or masked; half masked, ties; zeros of both signs and smallest numbers"""
    rng = np.random.default_rng(V)
    x = 2 * rng.standard_normal((8, V))
    x[0] -= x[0].max()
    x[1] = 0.0
    x[2], x[2, V // 2] = -3e4, 0.0
    x[3], x[3, 0] = -np.inf, 0.0
    x[4] = np.where(np.arange(V) % 2, -np.inf, np.minimum(x[4], 0.0))
    x[4, [0, V - 1 - (V - 1) % 2]] = 0.0
    x[5] = np.where(np.arange(V) % 3, -0.0, 0.0)
    x[6] = np.where(np.arange(V) % 3, np.nan, -np.inf)
    x[6, V - 1] = 0.0
    x[7] -= x[7].max()
    x[7, ::5] = -np.inf
    return x


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [3, 999, 5003, 50257])
@pytest.mark.parametrize("T", [1e-7, 1e-8, 4.2e-9, 1e-9, 1e-10, 1e-20, 1e-30, 1e-38, 1e-45])
def test_cold_rows_whose_largest_logit_is_zero(llma, dtype, V, T):  # noqa: F811
    x = torch.tensor(rows_at_zero(V), dtype=torch.float32).to(DT[dtype])
    if dtype != "fp16":
        x[2] = torch.where(x[2] == 0, x[2], torch.finfo(x.dtype).min)
    wide = torch.full((8, V + 3), 5.0, dtype=x.dtype, device="cuda")        # rows that begin and end inside a piece, larger logits on both sides
    wide[:, 1:V + 1] = x.cuda()
    tokens = np.random.default_rng(1).integers(0, V, 8)
    tokens[3] = 0
    t = np.full(8, T, np.float32)
    got = run(llma, wide[:, 1:V + 1], tokens, t, 5)
    for i in range(8):
        lp, rank, entropy, top, top_lp = mx.logprobs(x[i].double().numpy(), int(tokens[i]), float(t[i]), 5)
        # what counts is within 2^7 of the maximum in units of 2^x: 4 roundings of a term and one for each power of two of its argument, one for each level of a sum, as elsewhere; the
        # quotient by T and the result round once more.  Below fp32's range a log probability is minus infinity
        err = 2.0 ** -24 * (4 + 128 + 20)
        fp32 = lambda v: v if v >= -FLT_MAX else -np.inf
        assert near(got["logprob"][i], fp32(lp), err), (i, got["logprob"][i], lp)
        assert near(got["entropy"][i], entropy, 2 * err * (1 + min(entropy, 128.0))), (i, got["entropy"][i], entropy)
        assert got["rank"][i] == rank and got["top_tokens"][i].tolist() == top, i
        assert all(near(a, fp32(b), err) for a, b in zip(got["top_logprobs"][i], top_lp)), (i, got["top_logprobs"][i], top_lp)
