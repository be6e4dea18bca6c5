"""What the stateless calls of serving on pages refuse before any device work (no GPU needed): negative codes, a text, nothing enqueued."""
import ctypes

import pytest

import paper_2304_04487_amd as llma

P = 1 << 20                                     # an address that is 16-byte aligned; nothing follows it


@pytest.fixture(scope="module")
def lib():
    return llma.load_library()


def cache(**kw):
    return llma.PagedCacheC(**{**dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=4, n_kv_heads=2, head_dim=64), **kw})


MAP = dict(lens=P, rows=P, slots=None, n_seqs=2, n_slots=2, table=P, max_blocks=3, owned=P, free_pages=P, n_free=P, n_pages=6, row_offsets=P, lens_after=2 * P,
           slot_map=P, row_pos=P, max_rows=5, status=P, stream=None)
APPEND = dict(cache=None, k=P, v=P, dtype=1, k_row=64, k_head=64, v_row=64, v_head=64, slot_map=P, n_rows=3, stream=None)
ATTEND = dict(cache=None, q=P, dtype=1, n_heads=4, q_row=256, q_head=64, table=P, slots=None, n_slots=2, max_blocks=3, lens=P, row_offsets=P, n_seqs=2, n_rows=6,
              max_rows=3, scale=0.1, out=2 * P, out_row=256, out_head=64, work=P, work_bytes=1 << 30, stream=None)
VERIFY = dict(logits=P, dtype=0, row_stride=100, vocab=100, n_seqs=2, k=3, drafts=P, n_draft=None, draft_probs=None, temperature=None, u_accept=P, u_sample=P,
              n_accepted=P, next_token=P, emitted=P, work=P, work_bytes=1 << 30, stream=None)
I, R = llma.LLMA_E_INVAL, llma.LLMA_E_RANGE


def call(lib, name, base, change):
    a = {**base, **change}
    if "cache" in a:
        c = a["cache"] if a["cache"] is not None else cache()
        a["cache"] = ctypes.byref(c) if not isinstance(c, str) else None
    return getattr(lib, name)(*a.values())


@pytest.mark.parametrize("change,code", [
    (dict(lens=None), I), (dict(rows=None), I), (dict(table=None), I), (dict(owned=None), I), (dict(free_pages=None), I), (dict(n_free=None), I), (dict(row_offsets=None), I),
    (dict(lens_after=None), I), (dict(status=None), I), (dict(slot_map=None), I), (dict(row_pos=None), I), (dict(n_seqs=0), I), (dict(n_slots=0), I), (dict(max_blocks=0), I),
    (dict(n_pages=0), I), (dict(max_rows=-1), I), (dict(n_slots=65537), R), (dict(n_seqs=3), R), (dict(n_pages=1 << 25), R), (dict(max_blocks=1 << 25), R), (dict(lens_after=P), I), (dict(max_rows=(1 << 30) + 1), R)])
def test_map_pages(lib, change, code):
    assert call(lib, "llma_map_pages", MAP, change) == code
    assert b"llma_map_pages" in lib.llma_last_error(None)


@pytest.mark.parametrize("change,code", [
    (dict(cache="null"), I), (dict(cache=cache(k=None)), I), (dict(cache=cache(v_scale=None)), I), (dict(cache=cache(head_dim=96)), I), (dict(cache=cache(n_pages=0)), I),
    (dict(cache=cache(n_kv_heads=0)), I), (dict(cache=cache(n_kv_heads=1025)), I), (dict(cache=cache(n_pages=1 << 25)), R), (dict(cache=cache(v=P + 8)), I), (dict(k=None), I), (dict(v=None), I),
    (dict(slot_map=None), I), (dict(dtype=3), I), (dict(dtype=-1), I), (dict(n_rows=-1), I), (dict(k=P + 2), I), (dict(v_row=60), I), (dict(k_head=4), I), (dict(k_row=-64), I),
    (dict(cache=cache(n_kv_heads=1024), n_rows=1 << 24), R), (dict(n_rows=(1 << 28) + 1), R)])
def test_append_paged(lib, change, code):
    assert call(lib, "llma_append_paged", APPEND, change) == code
    assert b"llma_append_paged" in lib.llma_last_error(None)


@pytest.mark.parametrize("change,code", [
    (dict(cache="null"), I), (dict(cache=cache(head_dim=32)), I), (dict(q=None), I), (dict(out=None), I), (dict(table=None), I), (dict(lens=None), I), (dict(row_offsets=None), I), (dict(work=None), I),
    (dict(dtype=7), I), (dict(n_heads=3), I), (dict(n_heads=0), I), (dict(n_seqs=-1), I), (dict(n_rows=-1), I), (dict(max_rows=-1), I), (dict(max_blocks=0), I), (dict(n_seqs=4097), R),
    (dict(n_slots=1), R), (dict(slots=P, n_slots=0), R), (dict(max_blocks=1 << 25), R), (dict(max_rows=1 << 25), R), (dict(q=P + 8), I), (dict(out=P + 4), I), (dict(q_row=7), I), (dict(out_head=68), I),
    (dict(out=P), I), (dict(out_row=128), I), (dict(out_row=0), I), (dict(out_head=0), I), (dict(out_row=64, out_head=320), I), (dict(work_bytes=100), I), (dict(work=P + 4), I)])
def test_attend_paged(lib, change, code):
    assert call(lib, "llma_attend_paged", ATTEND, change) == code
    assert b"llma_attend_paged" in lib.llma_last_error(None)


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), I), (dict(drafts=None), I), (dict(u_accept=None), I), (dict(u_sample=None), I), (dict(n_accepted=None), I), (dict(next_token=None), I), (dict(emitted=None), I), (dict(work=None), I),
    (dict(dtype=5), I), (dict(n_seqs=-1), I), (dict(k=-1), I), (dict(vocab=0), I), (dict(k=64), R), (dict(vocab=(1 << 24) + 1, row_stride=1 << 25), R), (dict(n_seqs=(1 << 20) + 1), R), (dict(k=0, n_seqs=(1 << 22) + 1), R), (dict(row_stride=99), I),
    (dict(logits=P + 2), I), (dict(work_bytes=16), I), (dict(work=P + 8), I)])
def test_verify_sampled(lib, change, code):
    assert call(lib, "llma_verify_sampled", VERIFY, change) == code
    assert b"llma_verify_sampled" in lib.llma_last_error(None)


def test_out_with_heads_outermost_is_not_refused(lib):
    """(the next check is what refuses: a workspace that is too small)"""
    assert call(lib, "llma_attend_paged", ATTEND, dict(out_row=64, out_head=384, work_bytes=0)) == I
    assert b"workspace" in lib.llma_last_error(None)


def test_calls_without_rows_are_done_at_once(lib):
    assert call(lib, "llma_append_paged", APPEND, dict(n_rows=0, k=None, v=None, slot_map=None)) == 0
    for none in (dict(n_seqs=0), dict(n_rows=0), dict(max_rows=0)):
        assert call(lib, "llma_attend_paged", ATTEND, {**none, "q": None, "out": None}) == 0
    assert call(lib, "llma_verify_sampled", VERIFY, dict(n_seqs=0, logits=None)) == 0


def test_workspace_sizes(lib):
    assert lib.llma_attend_paged_workspace(1, 1, 8, 8, 64, 1) > 0
    assert lib.llma_attend_paged_workspace(1, 1, 8, 3, 64, 1) == I
    assert lib.llma_attend_paged_workspace(4097, 1, 8, 8, 64, 1) == R
    assert lib.llma_verify_sampled_workspace(1, 0, 1) > 0
    assert lib.llma_verify_sampled_workspace(1, 64, 100) == R


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    z = torch.zeros(4, dtype=torch.int32)
    pages = llma.PageTable(z.reshape(2, 2), z[:2], z, z[:1])
    with pytest.raises(llma.LlmaError) as e:
        llma.llma_map_pages(pages, z[:2], z[:2], z[:3], z[:2], None, None, z[:1])
    assert e.value.code == I and "device" in str(e.value)
    with pytest.raises(llma.LlmaError):
        llma.llma_append_paged(None, z, z, z)
    with pytest.raises(llma.LlmaError):
        llma.llma_attend_paged(None, z, z, z, z, 1, 1.0, z)
    with pytest.raises(llma.LlmaError):
        llma.llma_verify_sampled(z, z, z, z, z, z, z)


def test_sampled_steps_without_a_context(lib):
    f = (ctypes.c_float * 2)(0.5, 0.5)
    assert lib.llma_verify_step_sampled(None, 0, None, 0, 1.0, None, 0.5, None, None, None) == I
    assert lib.llma_verify_step_sampled_batch(None, 1, None, None, 0, f, f, f, None, None, None) == I
