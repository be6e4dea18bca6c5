"""Attention over pages refuses a scale that is no number: its kernels take the largest of the scale and a small number, which passes over NaN (no GPU needed)."""
import pytest

import paper_2304_04487_amd as llma
import test_mx_refusals as mx


@pytest.fixture(scope="module")
def lib():
    return llma.load_library()


def test_nan_is_refused(lib):
    nan = float("nan")
    assert mx.call(lib, "llma_attend_paged_mx", mx.ATTEND, dict(scale=nan)) == llma.LLMA_E_INVAL
    assert b"llma_attend_paged_mx: scale" in lib.llma_last_error(None)
    assert mx.call(lib, "llma_attend_paged", mx.ATTEND, dict(scale=nan)) == llma.LLMA_E_INVAL
    assert b"llma_attend_paged: scale" in lib.llma_last_error(None)
