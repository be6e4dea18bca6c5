"""llma_verify_sampled on rows of logits that lie in wider ones: any row stride, without drafts too, where the middle dimension has one entry and its stride says nothing."""
import numpy as np
import pytest
import torch

from test_gpu_sampled import DT, call, check, inputs, llma  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B", [1, 2, 7])
@pytest.mark.parametrize("V,W", [(999, 999), (999, 1024), (17, 4001)])
def test_rows_without_drafts(llma, dtype, B, V, W):  # noqa: F811
    logits, drafts, ua, us, _ = inputs(B, 0, V, dtype, V + B)
    wide = torch.full((B, W), 50.0, dtype=DT[dtype], device="cuda")
    wide[:, :V] = logits[:, 0]
    for view in (wide[:, :V][:, None, :], wide[:, None, :V], wide.as_strided((B, 1, V), (W, 0, 1)), wide.as_strided((B, 1, V), (W, 3, 1))):
        check(llma, view, drafts, ua, us)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_with_drafts(llma, dtype):  # noqa: F811
    """(and what stays refused: sequences whose rows are not one row stride after the other)"""
    V, W, B, k = 500, 777, 3, 2
    logits, drafts, ua, us, _ = inputs(B, k, V, dtype, 5)
    wide = torch.full((B, k + 2, W), 50.0, dtype=DT[dtype], device="cuda")
    wide[:, :k + 1, :V] = logits
    check(llma, wide[:, :k + 1].contiguous()[:, :, :V], drafts, ua, us)
    for b in range(B):
        check(llma, wide[b:b + 1, :k + 1, :V], drafts[b:b + 1], ua[b:b + 1], us[b:b + 1])
    with pytest.raises(llma.LlmaError) as e:
        call(llma, wide[:, :k + 1, :V], drafts, ua, us)
    assert e.value.code == llma.LLMA_E_INVAL and "stride" in str(e.value)
