"""Sampled steps on the host side alone (tests/host_stub.cpp): what a context refuses before any device work."""
import ctypes

import numpy as np

import paper_2304_04487_amd as llma
from test_host_calls import i32, lib  # noqa: F401


def test_a_model_of_more_tokens_than_sampling_takes(lib):  # noqa: F811
    """refused by the sampled step as by the stateless call; greedy steps run"""
    d, F, V = 64, 64, (1 << 24) + 16
    cfg = llma.ModelCfgC(1, d, 1, 64, F, V, 64, 1, 2, llma.LLMA_DTYPE_BF16, 1, 1e-6, 1e4)
    keep = np.zeros(V * d, np.uint16)
    p = keep.ctypes.data
    per = (ctypes.c_void_p * 1)(p)
    w, h = llma.WeightsC(p, p, p, per, per, per, per, per, per), ctypes.c_void_p()
    assert lib.llma_create(ctypes.byref(cfg), ctypes.byref(w), None, ctypes.byref(h)) == 0, lib.llma_last_error(None)
    assert lib.llma_prefill(h, 0, i32(1, 2, 3), 3) == 0
    enqueued = lib.stub_pending()
    f = (ctypes.c_float * 1)(0.5)
    assert lib.llma_verify_step_sampled(h, 0, i32(5), 1, ctypes.c_float(1.0), f, ctypes.c_float(0.5), None, None, None) == llma.LLMA_E_RANGE
    assert b"2^24" in lib.llma_last_error(h) and lib.stub_pending() == enqueued
    assert lib.llma_verify_step(h, 0, i32(5), 1, None, None, None) == 0
    assert lib.llma_destroy(h) == 0
