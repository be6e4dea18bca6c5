"""What the calls of the 4-bit cache, of reading pages and of token log probabilities refuse before any device work (no GPU needed), and the plain forms' own checks."""
import ctypes

import numpy as np
import pytest

import mx_oracle as mx
import paper_2304_04487_amd as llma

P = 1 << 20                                     # an address that is 16-byte aligned; nothing follows it
I, R = llma.LLMA_E_INVAL, llma.LLMA_E_RANGE


@pytest.fixture(scope="module")
def lib():
    return llma.load_library()


def cache(mx_format, **kw):
    return (llma.PagedMxCacheC if mx_format else llma.PagedCacheC)(**{**dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=4, n_kv_heads=2, head_dim=64), **kw})


APPEND = dict(cache={}, k=P, v=P, dtype=1, k_row=64, k_head=64, v_row=64, v_head=64, slot_map=P, n_rows=3, stream=None)
ATTEND = dict(cache={}, q=P, dtype=1, n_heads=4, q_row=256, q_head=64, table=P, slots=None, n_slots=2, max_blocks=3, lens=P, row_offsets=P, n_seqs=2, n_rows=6,
              max_rows=3, scale=0.1, out=2 * P, out_row=256, out_head=64, work=P, work_bytes=1 << 30, stream=None)
READ = dict(cache={}, table=P, slots=None, n_slots=2, max_blocks=3, first=None, row_offsets=P, n_seqs=2, n_rows=6, k=P, v=2 * P, dtype=1, k_row=128, k_head=64, v_row=64, v_head=384,
            stream=None)
LOGPROBS = dict(logits=P, dtype=0, row_stride=100, vocab=100, n_rows=3, tokens=P, temperature=None, n_top=2, logprob=P, rank=P, entropy=P, top_tokens=P, top_logprobs=P, work=P,
                work_bytes=1 << 30, stream=None)


def call(lib, name, base, change):
    a = {**base, **change}
    if "cache" in a:
        a["cache"] = ctypes.byref(cache(name.endswith("_mx"), **a["cache"])) if a["cache"] is not None else None
    return getattr(lib, name)(*a.values())


CACHE = [(dict(cache=None), I), (dict(cache=dict(k=None)), I), (dict(cache=dict(v_scale=None)), I), (dict(cache=dict(head_dim=96)), I), (dict(cache=dict(head_dim=32)), I),
         (dict(cache=dict(n_pages=0)), I), (dict(cache=dict(n_kv_heads=0)), I), (dict(cache=dict(n_kv_heads=1025)), I), (dict(cache=dict(n_pages=1 << 25)), R), (dict(cache=dict(v=P + 8)), I)]


@pytest.mark.parametrize("change,code", CACHE + [
    (dict(cache=dict(k_scale=P + 4)), I), (dict(cache=dict(v_scale=P + 8)), I), (dict(k=None), I), (dict(v=None), I),
    (dict(slot_map=None), I), (dict(dtype=3), I), (dict(dtype=-1), I), (dict(n_rows=-1), I), (dict(k=P + 2), I), (dict(v_row=60), I), (dict(k_head=4), I), (dict(k_row=-64), I),
    (dict(cache=dict(n_kv_heads=1024), n_rows=1 << 24), R), (dict(n_rows=(1 << 28) + 1), R)])
def test_append(lib, change, code):
    assert call(lib, "llma_append_paged_mx", APPEND, change) == code
    assert b"llma_append_paged_mx" in lib.llma_last_error(None)


@pytest.mark.parametrize("change,code", CACHE + [
    (dict(cache=dict(k_scale=P + 4)), I), (dict(q=None), I), (dict(out=None), I), (dict(table=None), I), (dict(lens=None), I), (dict(row_offsets=None), I), (dict(work=None), I),
    (dict(dtype=7), I), (dict(n_heads=3), I), (dict(n_heads=0), I), (dict(n_seqs=-1), I), (dict(n_rows=-1), I), (dict(max_rows=-1), I), (dict(max_blocks=0), I), (dict(n_seqs=4097), R),
    (dict(n_slots=1), R), (dict(slots=P, n_slots=0), R), (dict(max_blocks=1 << 25), R), (dict(max_rows=1 << 25), R), (dict(q=P + 8), I), (dict(out=P + 4), I), (dict(q_row=7), I), (dict(out_head=68), I),
    (dict(out=P), I), (dict(out_row=128), I), (dict(out_row=0), I), (dict(work=P + 8), I), (dict(work_bytes=16), I)])
def test_attend(lib, change, code):
    assert call(lib, "llma_attend_paged_mx", ATTEND, change) == code
    assert b"llma_attend_paged_mx" in lib.llma_last_error(None)


@pytest.mark.parametrize("name", ["llma_read_paged", "llma_read_paged_mx"])
@pytest.mark.parametrize("change,code", CACHE + [
    (dict(table=None), I), (dict(row_offsets=None), I), (dict(k=None), I), (dict(v=None), I), (dict(dtype=3), I), (dict(n_seqs=-1), I), (dict(n_rows=-1), I), (dict(max_blocks=0), I),
    (dict(n_seqs=4097), R), (dict(max_blocks=1 << 25), R), (dict(n_rows=(1 << 27) + 1), R), (dict(n_slots=1), R), (dict(slots=P, n_slots=0), R), (dict(k=P + 8), I), (dict(v=P + 4), I),
    (dict(k_row=100), I), (dict(v_head=-64), I), (dict(v=P), I), (dict(k_row=64), I), (dict(v_head=320), I), (dict(k_row=0), I)])
def test_read(lib, name, change, code):
    assert call(lib, name, READ, change) == code
    assert name.encode() in lib.llma_last_error(None)


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), I), (dict(work=None), I), (dict(tokens=None), I), (dict(tokens=None, logprob=None), I), (dict(tokens=None, rank=None), I), (dict(top_tokens=None), I), (dict(top_logprobs=None), I),
    (dict(n_rows=-1), I), (dict(vocab=0), I), (dict(n_top=-1), I), (dict(n_top=65), R), (dict(vocab=(1 << 24) + 1), R), (dict(n_rows=(1 << 22) + 1), R), (dict(n_rows=1 << 20, vocab=1 << 21), R),
    (dict(dtype=3), I), (dict(row_stride=99), I), (dict(row_stride=(1 << 40) + 1), I), (dict(logits=P + 1), I), (dict(work=P + 8), I), (dict(work_bytes=16), I)])
def test_logprobs(lib, change, code):
    assert call(lib, "llma_token_logprobs", LOGPROBS, change) == code
    assert b"llma_token_logprobs" in lib.llma_last_error(None)


def test_nothing_to_do_is_no_error(lib):
    for name, base, change in (("llma_append_paged_mx", APPEND, dict(n_rows=0)), ("llma_attend_paged_mx", ATTEND, dict(n_rows=0)), ("llma_attend_paged_mx", ATTEND, dict(n_seqs=0)),
                               ("llma_attend_paged_mx", ATTEND, dict(max_rows=0)), ("llma_read_paged", READ, dict(n_seqs=0)), ("llma_read_paged_mx", READ, dict(n_rows=0)),
                               ("llma_token_logprobs", LOGPROBS, dict(n_rows=0))):
        assert call(lib, name, base, change) == llma.LLMA_OK


def test_workspaces(lib):
    for bad in ((4097, 1, 8, 8, 64, 1), (1, 0, 8, 8, 64, 1), (1, 1, 8, 3, 64, 1), (1, 1, 8, 8, 32, 1)):
        assert lib.llma_attend_paged_mx_workspace(*bad) < 0
    # rises with everything that it depends on
    assert 0 < llma.llma_attend_paged_mx_workspace(1, 200, 8, 8, 64, 1) <= llma.llma_attend_paged_mx_workspace(16, 200, 8, 8, 64, 9)
    assert lib.llma_token_logprobs_workspace(1, 1, 65) < 0 and lib.llma_token_logprobs_workspace(1, 0, 0) < 0
    assert 0 < llma.llma_token_logprobs_workspace(9, 32000, 0) < llma.llma_token_logprobs_workspace(9, 32000, 1)


def test_tensors_that_are_none_are_refused():
    for fn, args in ((llma.llma_append_paged_mx, (None, [1], None, None)), (llma.llma_attend_paged_mx, (None, 3, None, None, None, 1, 1.0, None)),
                     (llma.llma_read_paged, (None, None, None, None, 3, None)), (llma.llma_read_paged_mx, (None, None, None, None, [1], None)), (llma.llma_token_logprobs, ([1.0], None, None))):
        with pytest.raises(llma.LlmaError):
            fn(*args)


def test_the_plain_encoding():
    """nearest codes, ties to even, by brute force over the grid; a scale of half the size would not do"""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * np.exp2(rng.integers(-70, 60, (200, 1)))
    x[5], x[6, :32] = 0, [7, -7, 5, 2.5, 3.5, 1.75, 1.25, 0.75, 0.25, -0.25] + [0] * 22
    codes, scale = mx.encode(x)
    got = mx.values(codes, scale)
    for i in range(200):
        for b in range(2):
            s, v = 2.0 ** (int(scale[i, b]) - 127), x[i, 32 * b:32 * b + 32]
            assert abs(v).max() <= 7 * s and (scale[i, b] == 63 or abs(v).max() > 3.5 * s)
            err = abs(got[i, 32 * b:32 * b + 32] - v)
            assert np.allclose(err, abs(v[:, None] - s * mx.VALUES).min(-1), rtol=1e-12, atol=0)
    assert got[6, :10].tolist() == [6, -6, 4, 2, 4, 2, 1, 1, 0, 0]
    assert mx.encode(np.array([[np.nan] + [1.0] * 31 + [np.inf] + [2.0] * 31]))[1].tolist() == [[255, 126]]


def test_a_workspace_for_many_sequences_does_for_fewer(lib):
    for blocks in (3, 60, 4000):
        for heads, kv, dh in ((32, 8, 128), (8, 8, 64), (64, 64, 128), (16, 1, 64), (600, 300, 128)):
            for rows in (1, 9, 65, 300, 2000):
                sizes = [llma.llma_attend_paged_mx_workspace(n, blocks, heads, kv, dh, rows) for n in (1, 2, 3, 7, 30, 64, 200)]
                assert sizes == sorted(sizes), (blocks, heads, kv, dh, rows, sizes)
                assert sizes[-1] < 70 << 20, (blocks, heads, kv, dh, rows, sizes)
