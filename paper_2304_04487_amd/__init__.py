"""Python binding of libllma.so (include/llma.h): argument marshalling only.

Every step of the decoding path runs inside the HIP library; PyTorch is used here only to
hold device memory (weights handed to llma_create, logits dump buffers) and to name the
stream.  There is no CPU fallback: if the shared library has not been built, importing the
functions works but the first call raises LlmaError.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_void_p

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libllma.so")

LLMA_OK, LLMA_E_INVAL, LLMA_E_RANGE, LLMA_E_NOMEM, LLMA_E_HIP, LLMA_E_STATE = 0, -1, -2, -3, -4, -5
LLMA_DTYPE_F32, LLMA_DTYPE_BF16 = 0, 1
LLMA_OPT_ACT_SPLIT, LLMA_OPT_KERNEL_TIMING, LLMA_OPT_USE_GRAPH = 1, 2, 3

EXPORTS = [
    "llma_create", "llma_destroy", "llma_last_error", "llma_reset", "llma_prefill", "llma_get_state",
    "llma_set_pending", "llma_kv_import", "llma_find_trigger", "llma_verify_step",
    "llma_verify_step_batch", "llma_generate", "llma_generate_batch", "llma_set_logits_dump", "llma_set_option",
    "llma_get_kernel_timing", "llma_time_ffn_gemm", "llma_time_step_gemm", "llma_device_bytes", "llma_find_trigger_static", "llma_truncate",
    "llma_describe", "llma_map_pages", "llma_append_paged", "llma_attend_paged", "llma_attend_paged_workspace",
    "llma_verify_sampled", "llma_verify_sampled_workspace", "llma_verify_step_sampled", "llma_verify_step_sampled_batch",
    "llma_read_paged", "llma_append_paged_mx", "llma_attend_paged_mx", "llma_attend_paged_mx_workspace", "llma_read_paged_mx",
    "llma_token_logprobs", "llma_token_logprobs_workspace",
]
LLMA_TRIGGER_STATIC_MAX_REF = 1 << 20
LLMA_DTYPE_F16, LLMA_KV_PAGED = 2, 2
LLMA_PAGE, LLMA_PAGED_MAX_SEQS, LLMA_SAMPLED_MAX_K, LLMA_LOGPROBS_MAX_TOP = 64, 4096, 63, 64


class LlmaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"llma error {code}: {msg}")
        self.code = code


class ModelCfgC(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("n_layers", "d_model", "n_heads", "head_dim", "d_ffn", "vocab",
                                       "max_seq", "max_batch", "max_k", "dtype", "kv_split")] + \
               [("rms_eps", c_float), ("rope_theta", c_float)]


class WeightsC(ctypes.Structure):
    _fields_ = [("embed", c_void_p), ("lm_head", c_void_p), ("final_norm", c_void_p),
                ("wqkv", POINTER(c_void_p)), ("wo", POINTER(c_void_p)), ("wgu", POINTER(c_void_p)),
                ("wdown", POINTER(c_void_p)), ("norm1", POINTER(c_void_p)), ("norm2", POINTER(c_void_p))]


class PagedCacheC(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("k_scale", c_void_p), ("v_scale", c_void_p),
                ("n_pages", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32)]


class PagedMxCacheC(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("k_scale", c_void_p), ("v_scale", c_void_p),
                ("n_pages", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32)]


class StepRec(ctypes.Structure):
    _fields_ = [("rows_in", c_int32), ("emitted", c_int32), ("doc", c_int32), ("pos", c_int32)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads the in-tree libllma.so; raises LlmaError when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise LlmaError(LLMA_E_INVAL, f"{LIB_PATH} is missing: run `python -m paper_2304_04487_amd.build` "
                                      "(or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    i32p, vp = POINTER(c_int32), c_void_p
    lib.llma_create.argtypes = [POINTER(ModelCfgC), POINTER(WeightsC), vp, POINTER(vp)]
    lib.llma_destroy.argtypes = [vp]
    lib.llma_last_error.argtypes = [vp]
    lib.llma_last_error.restype = c_char_p
    lib.llma_reset.argtypes = [vp, c_int32]
    lib.llma_prefill.argtypes = [vp, c_int32, i32p, c_int32]
    lib.llma_get_state.argtypes = [vp, c_int32, i32p, i32p]
    lib.llma_set_pending.argtypes = [vp, c_int32, c_int32]
    lib.llma_truncate.argtypes = [vp, c_int32, c_int32]
    lib.llma_kv_import.argtypes = [vp, c_int32, c_int32, vp, vp, c_int32]
    lib.llma_find_trigger.argtypes = [i32p, c_int32, i32p, i32p, c_int32, c_int32, i32p, i32p]
    lib.llma_find_trigger_static.argtypes = [vp, c_int32, vp, c_int32, vp, c_int32, c_int32, vp, vp]
    lib.llma_verify_step.argtypes = [vp, c_int32, i32p, c_int32, i32p, i32p, i32p]
    lib.llma_verify_step_batch.argtypes = [vp, c_int32, i32p, i32p, c_int32, i32p, i32p, i32p]
    lib.llma_verify_step_sampled.argtypes = [vp, c_int32, i32p, c_int32, c_float, POINTER(c_float), c_float, i32p, i32p, i32p]
    lib.llma_verify_step_sampled_batch.argtypes = [vp, c_int32, i32p, i32p, c_int32, POINTER(c_float), POINTER(c_float), POINTER(c_float), i32p, i32p, i32p]
    lib.llma_generate.argtypes = [vp, c_int32, i32p, c_int32, i32p, i32p, c_int32, c_int32, c_int32, c_int32,
                                  i32p, i32p, POINTER(StepRec), i32p]
    lib.llma_generate_batch.argtypes = [vp, c_int32, i32p, i32p, i32p, i32p, i32p, i32p, c_int32, c_int32, c_int32,
                                        i32p, i32p, POINTER(StepRec), i32p]
    lib.llma_set_logits_dump.argtypes = [vp, vp, c_int32]
    lib.llma_set_option.argtypes = [vp, c_int32, c_int32]
    lib.llma_get_kernel_timing.argtypes = [vp, POINTER(c_int64), POINTER(c_double)]
    lib.llma_time_ffn_gemm.argtypes = [vp, c_int32, c_int32, POINTER(c_double)]
    lib.llma_time_step_gemm.argtypes = [vp, c_int32, c_int32, c_int32, POINTER(c_double)]
    lib.llma_map_pages.argtypes = [vp, vp, vp, c_int32, c_int32, vp, c_int32, vp, vp, vp, c_int32, vp, vp, vp, vp, c_int32, vp, vp]
    lib.llma_append_paged.argtypes = [POINTER(PagedCacheC), vp, vp, c_int32, c_int64, c_int64, c_int64, c_int64, vp, c_int32, vp]
    lib.llma_append_paged_mx.argtypes = [POINTER(PagedMxCacheC)] + lib.llma_append_paged.argtypes[1:]
    lib.llma_attend_paged_workspace.argtypes = lib.llma_attend_paged_mx_workspace.argtypes = [c_int32] * 6
    lib.llma_attend_paged_workspace.restype = lib.llma_attend_paged_mx_workspace.restype = c_int64
    lib.llma_attend_paged.argtypes = [POINTER(PagedCacheC), vp, c_int32, c_int32, c_int64, c_int64, vp, vp, c_int32, c_int32, vp, vp,
                                      c_int32, c_int32, c_int32, c_float, vp, c_int64, c_int64, vp, c_int64, vp]
    lib.llma_attend_paged_mx.argtypes = [POINTER(PagedMxCacheC)] + lib.llma_attend_paged.argtypes[1:]
    lib.llma_read_paged.argtypes = [POINTER(PagedCacheC), vp, vp, c_int32, c_int32, vp, vp, c_int32, c_int32, vp, vp, c_int32, c_int64, c_int64, c_int64, c_int64, vp]
    lib.llma_read_paged_mx.argtypes = [POINTER(PagedMxCacheC)] + lib.llma_read_paged.argtypes[1:]
    lib.llma_token_logprobs_workspace.argtypes = [c_int32] * 3
    lib.llma_token_logprobs_workspace.restype = c_int64
    lib.llma_token_logprobs.argtypes = [vp, c_int32, c_int64, c_int32, c_int32, vp, vp, c_int32, vp, vp, vp, vp, vp, vp, c_int64, vp]
    lib.llma_verify_sampled_workspace.argtypes = [c_int32] * 3
    lib.llma_verify_sampled_workspace.restype = c_int64
    lib.llma_verify_sampled.argtypes = [vp, c_int32, c_int64, c_int32, c_int32, c_int32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, c_int64, vp]
    lib.llma_describe.argtypes = [vp, c_char_p, c_int32]
    lib.llma_device_bytes.argtypes = [vp]
    lib.llma_device_bytes.restype = c_int64
    _lib = lib
    return lib


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32).reshape(-1))


def _ptr(a: np.ndarray):
    """an int32 array as a call's POINTER(c_int32) argument; through the buffer where it has one that ctypes takes
    (0.3 us; data_as, for empty and read-only arrays, 2.5 us)"""
    try:
        return byref(c_int32.from_buffer(a))
    except (TypeError, ValueError):
        return a.ctypes.data_as(POINTER(c_int32))


def _check(rc: int, ctx=None) -> int:
    if rc < 0:
        raise LlmaError(rc, load_library().llma_last_error(ctx).decode())
    return rc


def llma_find_trigger(y, ref, doc_offsets, n: int):
    """Returns (matched, doc, pos); see llma_find_trigger in llma.h."""
    lib = load_library()
    y, ref, offs = _i32(y), _i32(ref), _i32(doc_offsets)
    doc, pos = c_int32(-1), c_int32(-1)
    rc = _check(lib.llma_find_trigger(_ptr(y), len(y), _ptr(ref), _ptr(offs), len(offs) - 1, n, byref(doc), byref(pos)))
    return bool(rc), doc.value, pos.value


def llma_find_trigger_static(y_dev, ref_dev, doc_offsets_dev, n: int, result_dev, stream=None):
    """The allocation-free trigger scan on DEVICE int32 tensors (anything with data_ptr() and
    numel()); result_dev: 3 device ints (matched, doc, pos).  Enqueues on `stream` (an object with
    .cuda_stream, or None for the default stream) and returns without synchronising."""
    lib = load_library()
    n_docs = max(int(doc_offsets_dev.numel()) - 1, 0)
    st = c_void_p(stream.cuda_stream) if stream is not None else None
    _check(lib.llma_find_trigger_static(c_void_p(y_dev.data_ptr()), int(y_dev.numel()), c_void_p(ref_dev.data_ptr()),
                                        int(ref_dev.numel()), c_void_p(doc_offsets_dev.data_ptr()), n_docs, n,
                                        c_void_p(result_dev.data_ptr()), st))


# ---- serving on pages: device tensors, a stream, no wait (see llma.h) --------------------------------------------------
class PagedCache:
    """A layer's cache: uint8 tensors k [n_pages, n_kv_heads, 64, head_dim] and v [n_pages, n_kv_heads, head_dim, 64], fp32
    k_scale and v_scale [n_pages, n_kv_heads]."""
    __slots__ = ("k", "v", "k_scale", "v_scale")

    def __init__(self, k, v, k_scale, v_scale):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, device="cuda"):
        import torch
        return cls(torch.empty((n_pages, n_kv_heads, LLMA_PAGE, head_dim), dtype=torch.uint8, device=device),
                   torch.empty((n_pages, n_kv_heads, head_dim, LLMA_PAGE), dtype=torch.uint8, device=device),
                   torch.empty((n_pages, n_kv_heads), dtype=torch.float32, device=device),
                   torch.empty((n_pages, n_kv_heads), dtype=torch.float32, device=device))


class PagedMxCache:
    """A layer's cache in 4 bits: uint8 tensors k [n_pages, n_kv_heads, 64, head_dim / 2], v [n_pages, n_kv_heads, head_dim / 2, 64], k_scale and v_scale
    [n_pages, n_kv_heads, head_dim / 32, 64] (see llma.h)."""
    __slots__ = ("k", "v", "k_scale", "v_scale")

    def __init__(self, k, v, k_scale, v_scale):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, device="cuda"):
        import torch
        u8 = {"dtype": torch.uint8, "device": device}
        return cls(torch.empty((n_pages, n_kv_heads, LLMA_PAGE, head_dim // 2), **u8), torch.empty((n_pages, n_kv_heads, head_dim // 2, LLMA_PAGE), **u8),
                   torch.empty((n_pages, n_kv_heads, head_dim // 32, LLMA_PAGE), **u8), torch.empty((n_pages, n_kv_heads, head_dim // 32, LLMA_PAGE), **u8))


class PageTable:
    """Who has which page: int32 tensors table [n_slots, max_blocks], owned [n_slots], free_pages [n_pages], n_free [1]."""
    __slots__ = ("table", "owned", "free_pages", "n_free")

    def __init__(self, table, owned, free_pages, n_free):
        self.table, self.owned, self.free_pages, self.n_free = table, owned, free_pages, n_free

    @classmethod
    def empty(cls, n_slots: int, max_blocks: int, n_pages: int, device="cuda"):
        """All pages free; page 0 is granted first."""
        import torch
        return cls(torch.full((n_slots, max_blocks), -1, dtype=torch.int32, device=device), torch.zeros(n_slots, dtype=torch.int32, device=device),
                   torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device), torch.full((1,), n_pages, dtype=torch.int32, device=device))


def _refuse(msg: str):
    raise LlmaError(LLMA_E_INVAL, msg)


_torch = None
_ROW_TYPES = {}


def _import_torch():
    global _torch
    import torch
    _ROW_TYPES.update({torch.bfloat16: LLMA_DTYPE_BF16, torch.float16: LLMA_DTYPE_F16, torch.float32: LLMA_DTYPE_F32})
    _torch = torch


class _Call:
    """Checks a call's tensors -- all on one device, of the type and shape they should have -- and names its stream.  The kernels of the smallest calls take a few
    microseconds, so what is asked of a tensor is asked in one line each (attend: 20 us a call with the stream looked up as an object and loops over shapes)."""
    __slots__ = ("who", "device", "given", "stream", "lib")

    def __init__(self, who: str, first, stream):
        if _torch is None:
            _import_torch()
        self.who = who
        if not isinstance(first, _torch.Tensor) or not first.is_cuda:
            _refuse(f"{who}: device tensors are wanted")
        self.lib = _lib or load_library()
        self.device = first.device
        self.given = stream
        if stream is None:
            self.stream = _torch._C._cuda_getCurrentRawStream(self.device.index)
        else:
            if getattr(stream, "device", self.device) != self.device:
                _refuse(f"{who}: the stream is not on the tensors' device")
            self.stream = stream.cuda_stream

    def ptr(self, name, t, dtype, shape):
        """a contiguous tensor's address"""
        if not isinstance(t, _torch.Tensor):
            _refuse(f"{self.who}: {name} has to be a tensor")
        if t.dtype is dtype and t.shape == shape and t.device == self.device and t.is_contiguous():
            return t.data_ptr()
        _refuse(f"{self.who}: {name} has to be a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")

    def rows(self, name, t, shape):
        """(address, dtype code) of rows whose features lie together, any other strides"""
        if not isinstance(t, _torch.Tensor):
            _refuse(f"{self.who}: {name} has to be a tensor")
        code = _ROW_TYPES.get(t.dtype)
        if code is not None and t.shape == shape and t.device == self.device and (t.stride(-1) == 1 or t.numel() == 0):
            return t.data_ptr(), code
        _refuse(f"{self.who}: {name} has to be a bf16, fp16 or fp32 tensor of shape {tuple(shape)} on {self.device} whose features lie together, not {t.dtype} {tuple(t.shape)}, "
                f"strides {t.stride()}, on {t.device}")

    def cache(self, c):
        k, u8, f32 = c.k, _torch.uint8, _torch.float32
        if k.dim() != 4:
            _refuse(f"{self.who}: cache.k has to be [n_pages, n_kv_heads, {LLMA_PAGE}, head_dim]")
        P, H, _, D = k.shape
        return PagedCacheC(self.ptr("cache.k", k, u8, (P, H, LLMA_PAGE, D)), self.ptr("cache.v", c.v, u8, (P, H, D, LLMA_PAGE)),
                           self.ptr("cache.k_scale", c.k_scale, f32, (P, H)), self.ptr("cache.v_scale", c.v_scale, f32, (P, H)), P, H, D)

    def mx_cache(self, c):
        k, u8 = c.k, _torch.uint8
        if k.dim() != 4:
            _refuse(f"{self.who}: cache.k has to be [n_pages, n_kv_heads, {LLMA_PAGE}, head_dim / 2]")
        P, H, _, D = k.shape
        scales = (P, H, D // 16, LLMA_PAGE)
        return PagedMxCacheC(self.ptr("cache.k", k, u8, (P, H, LLMA_PAGE, D)), self.ptr("cache.v", c.v, u8, (P, H, D, LLMA_PAGE)),
                             self.ptr("cache.k_scale", c.k_scale, u8, scales), self.ptr("cache.v_scale", c.v_scale, u8, scales), P, H, 2 * D)

    def workspace(self, given, size: int):
        """a workspace of the caller's, or one that lives until the stream has used it (the allocator orders its reuse on the stream)"""
        _check(size)
        if given is not None:
            if given.device != self.device or not given.is_contiguous():
                _refuse(f"{self.who}: workspace has to be a contiguous tensor on {self.device}")
            return given, given.numel() * given.element_size()
        if self.given is None:
            return _torch.empty(size, dtype=_torch.uint8, device=self.device), size
        with _torch.cuda.stream(self.given):
            return _torch.empty(size, dtype=_torch.uint8, device=self.device), size

    def run(self, fn, *args):
        if self.device.index == _torch.cuda.current_device():
            rc = fn(*args, self.stream)
        else:
            with _torch.cuda.device(self.device):
                rc = fn(*args, self.stream)
        if rc < 0:
            _check(rc)


def llma_map_pages(pages, lens, rows, row_offsets, lens_after, slot_map, row_pos, status, slots=None, stream=None):
    """Pages and slots of a step from the sequences' lengths (see llma.h).  pages: a PageTable; int32 tensors lens [n_slots],
    rows [n_seqs], slots [n_seqs] or None; written: row_offsets [n_seqs + 1], lens_after [n_seqs], slot_map and row_pos [max_rows] (or both None), status [1].
    Enqueues on `stream` (None: torch's current stream of the tensors' device) and returns without synchronising."""
    c = _Call("llma_map_pages", lens, stream)
    i32, p = _torch.int32, c.ptr
    S, blocks = pages.table.shape if pages.table.dim() == 2 else (-1, -1)
    B, P = rows.numel(), pages.free_pages.numel()
    if (slot_map is None) != (row_pos is None):
        _refuse("llma_map_pages: slot_map and row_pos come together")
    n = 0 if slot_map is None else slot_map.numel()
    c.run(c.lib.llma_map_pages, p("lens", lens, i32, (S,)), p("rows", rows, i32, (B,)), None if slots is None else p("slots", slots, i32, (B,)), B, S,
          p("pages.table", pages.table, i32, (S, blocks)), blocks, p("pages.owned", pages.owned, i32, (S,)), p("pages.free_pages", pages.free_pages, i32, (P,)),
          p("pages.n_free", pages.n_free, i32, (1,)), P, p("row_offsets", row_offsets, i32, (B + 1,)), p("lens_after", lens_after, i32, (B,)),
          None if n == 0 else p("slot_map", slot_map, i32, (n,)), None if n == 0 else p("row_pos", row_pos, i32, (n,)), n, p("status", status, i32, (1,)))


def _append(c, fn, d, k, v, slot_map):
    shape = (slot_map.numel(), d.n_kv_heads, d.head_dim)
    kp, kt = c.rows("k", k, shape)
    vp, vt = c.rows("v", v, shape)
    if kt != vt:
        _refuse(f"{c.who}: k and v have different types")
    c.run(fn, byref(d), kp, vp, kt, k.stride(0), k.stride(1), v.stride(0), v.stride(1), c.ptr("slot_map", slot_map, _torch.int32, (shape[0],)), shape[0])


def llma_append_paged(cache, k, v, slot_map, stream=None):
    """Writes rows k, v [n_rows, n_kv_heads, head_dim] (bf16, fp16 or fp32; features together, other strides as they are) into the paged
    cache at slot_map (int32 [n_rows], negative: nowhere); see llma.h.  Enqueues and returns without synchronising."""
    c = _Call("llma_append_paged", k, stream)
    _append(c, c.lib.llma_append_paged, c.cache(cache), k, v, slot_map)


def llma_append_paged_mx(cache, k, v, slot_map, stream=None):
    """The same into a PagedMxCache (4 bits; see llma.h)."""
    c = _Call("llma_append_paged_mx", k, stream)
    _append(c, c.lib.llma_append_paged_mx, c.mx_cache(cache), k, v, slot_map)


def _attend(c, fn, size, d, q, table, lens, row_offsets, max_rows, scale, out, slots, workspace):
    i32, p = _torch.int32, c.ptr
    shape = (q.shape[0], q.shape[1], d.head_dim) if q.dim() == 3 else (-1,)
    qp, qt = c.rows("q", q, shape)
    op, ot = c.rows("out", out, shape)
    if qt != ot:
        _refuse(f"{c.who}: out and q have different types")
    B = lens.numel()
    S, blocks = table.shape if table.dim() == 2 else (-1, -1)
    tp = p("table", table, i32, (S, blocks))
    ws, size = c.workspace(workspace, size(B, blocks, shape[1], d.n_kv_heads, d.head_dim, max_rows))
    c.run(fn, byref(d), qp, qt, shape[1], q.stride(0), q.stride(1), tp, None if slots is None else p("slots", slots, i32, (B,)),
          S, blocks, p("lens", lens, i32, (B,)), p("row_offsets", row_offsets, i32, (B + 1,)), B, shape[0], max_rows, scale,
          op, out.stride(0), out.stride(1), ws.data_ptr(), size)
    return out


def llma_attend_paged(cache, q, table, lens, row_offsets, max_rows: int, scale: float, out, slots=None, workspace=None, stream=None):
    """Causal attention of rows q [n_rows, n_heads, head_dim] over the paged cache into out (see llma.h).  int32 tensors table
    [n_slots, max_blocks], lens [n_seqs] (the step's rows included), row_offsets [n_seqs + 1], slots [n_seqs] or None; max_rows: no sequence has more
    rows.  workspace: at least llma_attend_paged_workspace() bytes of device memory, None: allocated for the call.  Enqueues
    and returns without synchronising.  Returns out."""
    c = _Call("llma_attend_paged", q, stream)
    return _attend(c, c.lib.llma_attend_paged, c.lib.llma_attend_paged_workspace, c.cache(cache), q, table, lens, row_offsets, max_rows, scale, out, slots, workspace)


def llma_attend_paged_workspace(n_seqs: int, max_blocks: int, n_heads: int, n_kv_heads: int, head_dim: int, max_rows: int) -> int:
    return _check(load_library().llma_attend_paged_workspace(n_seqs, max_blocks, n_heads, n_kv_heads, head_dim, max_rows))


def llma_attend_paged_mx(cache, q, table, lens, row_offsets, max_rows: int, scale: float, out, slots=None, workspace=None, stream=None):
    """The same over a PagedMxCache (4 bits; see llma.h).  workspace: at least llma_attend_paged_mx_workspace() bytes."""
    c = _Call("llma_attend_paged_mx", q, stream)
    return _attend(c, c.lib.llma_attend_paged_mx, c.lib.llma_attend_paged_mx_workspace, c.mx_cache(cache), q, table, lens, row_offsets, max_rows, scale, out, slots, workspace)


def llma_attend_paged_mx_workspace(n_seqs: int, max_blocks: int, n_heads: int, n_kv_heads: int, head_dim: int, max_rows: int) -> int:
    return _check(load_library().llma_attend_paged_mx_workspace(n_seqs, max_blocks, n_heads, n_kv_heads, head_dim, max_rows))


def _read(c, fn, d, table, first, row_offsets, k, v, slots):
    i32, p = _torch.int32, c.ptr
    shape = (k.shape[0] if k.dim() == 3 else -1, d.n_kv_heads, d.head_dim)
    kp, kt = c.rows("k", k, shape)
    vp, vt = c.rows("v", v, shape)
    if kt != vt:
        _refuse(f"{c.who}: k and v have different types")
    B = row_offsets.numel() - 1
    S, blocks = table.shape if table.dim() == 2 else (-1, -1)
    c.run(fn, byref(d), p("table", table, i32, (S, blocks)), None if slots is None else p("slots", slots, i32, (B,)), S, blocks,
          None if first is None else p("first", first, i32, (B,)), p("row_offsets", row_offsets, i32, (B + 1,)), B, shape[0], kp, vp, kt,
          k.stride(0), k.stride(1), v.stride(0), v.stride(1))


def llma_read_paged(cache, table, first, row_offsets, k, v, slots=None, stream=None):
    """Rows out of the paged cache into k, v [n_rows, n_kv_heads, head_dim] (bf16, fp16 or fp32; features together, other strides as they are): rows
    row_offsets[b] .. row_offsets[b + 1] - 1 become the positions from first[b] on of sequence b (see llma.h).  int32 tensors table [n_slots, max_blocks], first
    [n_seqs] (None: 0), row_offsets [n_seqs + 1], slots [n_seqs] or None.  Enqueues and returns without synchronising."""
    c = _Call("llma_read_paged", k, stream)
    _read(c, c.lib.llma_read_paged, c.cache(cache), table, first, row_offsets, k, v, slots)


def llma_read_paged_mx(cache, table, first, row_offsets, k, v, slots=None, stream=None):
    """The same out of a PagedMxCache (4 bits; see llma.h)."""
    c = _Call("llma_read_paged_mx", k, stream)
    _read(c, c.lib.llma_read_paged_mx, c.mx_cache(cache), table, first, row_offsets, k, v, slots)


def llma_verify_sampled(logits, drafts, u_accept, u_sample, n_accepted, next_token, emitted, n_draft=None, draft_probs=None, temperature=None,
                        workspace=None, stream=None):
    """Verifies drafts against the target's probabilities with given random numbers (see llma.h).  logits [n_seqs, k + 1, vocab] (bf16, fp16 or fp32, rows any
    stride apart), drafts int32 [n_seqs, k], u_accept fp32 [n_seqs, k], u_sample fp32 [n_seqs], n_draft int32 [n_seqs], draft_probs fp32
    [n_seqs, k, vocab], temperature fp32 [n_seqs]; written, int32: n_accepted, next_token [n_seqs], emitted [n_seqs, k + 1].  workspace: at least
    llma_verify_sampled_workspace() bytes of device memory, None: allocated for the call.  Enqueues and returns without synchronising."""
    c = _Call("llma_verify_sampled", logits, stream)
    i32, f32, p = _torch.int32, _torch.float32, c.ptr
    shape = logits.shape if logits.dim() == 3 else (-1, 0, -1)
    lp, lt = c.rows("logits", logits, shape)
    B, k, V = shape[0], shape[1] - 1, shape[2]
    if k < 0 or (B > 1 and k > 0 and logits.stride(0) != (k + 1) * logits.stride(1)):
        _refuse("llma_verify_sampled: logits has to be [n_seqs, k + 1, vocab] with all rows the same stride apart")
    row = logits.stride(1) if k > 0 else logits.stride(0)
    ws, size = c.workspace(workspace, c.lib.llma_verify_sampled_workspace(B, k, V))
    c.run(c.lib.llma_verify_sampled, lp, lt, row if B * (k + 1) > 1 else max(row, V), V, B, k, p("drafts", drafts, i32, (B, k)),
          None if n_draft is None else p("n_draft", n_draft, i32, (B,)), None if draft_probs is None else p("draft_probs", draft_probs, f32, (B, k, V)),
          None if temperature is None else p("temperature", temperature, f32, (B,)), p("u_accept", u_accept, f32, (B, k)), p("u_sample", u_sample, f32, (B,)),
          p("n_accepted", n_accepted, i32, (B,)), p("next_token", next_token, i32, (B,)), p("emitted", emitted, i32, (B, k + 1)), ws.data_ptr(), size)


def llma_verify_sampled_workspace(n_seqs: int, k: int, vocab: int) -> int:
    return _check(load_library().llma_verify_sampled_workspace(n_seqs, k, vocab))


def llma_token_logprobs(logits, tokens, logprob, rank=None, entropy=None, top_tokens=None, top_logprobs=None, temperature=None, workspace=None, stream=None):
    """Log probabilities of given tokens under softmax(logits / temperature), with ranks, entropy and the likeliest alternatives (see llma.h).  logits [n_rows, vocab]
    (bf16, fp16 or fp32, rows any stride apart), tokens int32 [n_rows] (or None), temperature fp32 [n_rows]; written, each may be None: logprob, entropy fp32 [n_rows],
    rank int32 [n_rows], top_tokens int32 and top_logprobs fp32 [n_rows, n_top] (both or none).  workspace: at least llma_token_logprobs_workspace() bytes
    of device memory, None: allocated for the call.  Enqueues and returns without synchronising."""
    c = _Call("llma_token_logprobs", logits, stream)
    i32, f32, p = _torch.int32, _torch.float32, c.ptr
    shape = logits.shape if logits.dim() == 2 else (-1, -1)
    lp, lt = c.rows("logits", logits, shape)
    n, V = shape
    if (top_tokens is None) != (top_logprobs is None):
        _refuse("llma_token_logprobs: top_tokens and top_logprobs come together")
    top = 0 if top_tokens is None else top_tokens.shape[-1] if top_tokens.dim() == 2 else -1
    ws, size = c.workspace(workspace, c.lib.llma_token_logprobs_workspace(n, V, top))
    c.run(c.lib.llma_token_logprobs, lp, lt, logits.stride(0) if n > 1 else max(logits.stride(0), V), V, n, None if tokens is None else p("tokens", tokens, i32, (n,)),
          None if temperature is None else p("temperature", temperature, f32, (n,)), top, None if logprob is None else p("logprob", logprob, f32, (n,)),
          None if rank is None else p("rank", rank, i32, (n,)), None if entropy is None else p("entropy", entropy, f32, (n,)),
          None if top == 0 else p("top_tokens", top_tokens, i32, (n, top)), None if top == 0 else p("top_logprobs", top_logprobs, f32, (n, top)), ws.data_ptr(), size)


def llma_token_logprobs_workspace(n_rows: int, vocab: int, n_top: int) -> int:
    return _check(load_library().llma_token_logprobs_workspace(n_rows, vocab, n_top))


class Context:
    """Owns one llma_ctx.  `cfg` is any object with n_layers, d_model, n_heads, head_dim, d_ffn,
    vocab, dtype ("fp32" | "bf16"), rms_eps, rope_theta; `weights` the dict of numpy arrays
    (bf16 as uint16 bit patterns) laid out as llma.h describes.  kv_paged: the cache as 8-bit pages (bf16 models) in place of
    the planes that kv_split names."""

    def __init__(self, cfg, weights: dict, max_seq: int, max_batch: int = 1, max_k: int = 16, device="cuda:0",
                 kv_split: bool = True, kv_paged: bool = False):
        import torch
        self._torch = torch
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        self.max_seq, self.max_batch, self.max_k = max_seq, max_batch, max_k
        self._h = c_void_p()
        torch.cuda.set_device(self.device)
        stream = torch.cuda.current_stream(self.device)
        L = len(weights["layers"])
        c = ModelCfgC(L, cfg.d_model, cfg.n_heads, cfg.head_dim, cfg.d_ffn, cfg.vocab, max_seq, max_batch, max_k,
                      LLMA_DTYPE_BF16 if cfg.dtype == "bf16" else LLMA_DTYPE_F32, LLMA_KV_PAGED if kv_paged else int(bool(kv_split)),
                      cfg.rms_eps, cfg.rope_theta)

        def dev(a):
            return torch.from_numpy(np.ascontiguousarray(a)).to(self.device)

        # upload layer by layer and let llma_create copy; the temporaries are freed afterwards
        keep = {"embed": dev(weights["embed"]), "lm_head": dev(weights["lm_head"]), "final_norm": dev(weights["final_norm"])}
        names = ("wqkv", "wo", "wgu", "wd", "norm1", "norm2")
        per = {n: [dev(lw[n]) for lw in weights["layers"]] for n in names}
        arr = {n: (c_void_p * L)(*[t.data_ptr() for t in per[n]]) for n in names}
        w = WeightsC(keep["embed"].data_ptr(), keep["lm_head"].data_ptr(), keep["final_norm"].data_ptr(),
                     arr["wqkv"], arr["wo"], arr["wgu"], arr["wd"], arr["norm1"], arr["norm2"])
        torch.cuda.synchronize(self.device)
        _check(self.lib.llma_create(byref(c), byref(w), c_void_p(stream.cuda_stream), byref(self._h)))
        del keep, per
        self._dump = None

    # -- lifetime
    def close(self):
        if self._h:
            self.lib.llma_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ck(self, rc):
        return _check(rc, self._h)

    # -- state
    def reset(self, seq: int = 0):
        self._ck(self.lib.llma_reset(self._h, seq))

    def prefill(self, prompt, seq: int = 0):
        p = _i32(prompt)
        self._ck(self.lib.llma_prefill(self._h, seq, _ptr(p), len(p)))

    def get_state(self, seq: int = 0):
        t, p = c_int32(), c_int32()
        self._ck(self.lib.llma_get_state(self._h, seq, byref(t), byref(p)))
        return t.value, p.value

    def truncate(self, new_len: int, seq: int = 0):
        self._ck(self.lib.llma_truncate(self._h, seq, int(new_len)))

    def set_pending(self, token: int, seq: int = 0):
        self._ck(self.lib.llma_set_pending(self._h, seq, int(token)))

    def kv_import(self, seq: int, layer: int, k_dev, v_dev, length: int):
        """k_dev, v_dev: torch device tensors, plain [n_heads, length, head_dim] in the model dtype
        (bf16 tensors or uint16 bit patterns for bf16 models)."""
        self._ck(self.lib.llma_kv_import(self._h, seq, layer, c_void_p(k_dev.data_ptr()), c_void_p(v_dev.data_ptr()), length))

    # -- the method
    def verify_step(self, draft, seq: int = 0):
        """Returns (n_accepted, next_token, emitted list)."""
        d = _i32(draft)
        k = len(d)
        na, nt = c_int32(), c_int32()
        em = np.zeros(k + 1, dtype=np.int32)
        self._ck(self.lib.llma_verify_step(self._h, seq, _ptr(d), k, byref(na), byref(nt), _ptr(em)))
        return na.value, nt.value, em[:na.value + 1].tolist()

    def verify_step_batch(self, seqs, drafts):
        """drafts: [n_seqs, k].  Returns (n_accepted[n_seqs], next_token[n_seqs], emitted[n_seqs][...])."""
        s = _i32(seqs)
        d2 = np.asarray(drafts, dtype=np.int32).reshape(len(s), -1)
        k = d2.shape[1]
        d = _i32(d2)
        na, nt = np.zeros(len(s), np.int32), np.zeros(len(s), np.int32)
        em = np.zeros(len(s) * (k + 1), np.int32)
        self._ck(self.lib.llma_verify_step_batch(self._h, len(s), _ptr(s), _ptr(d), k, _ptr(na), _ptr(nt), _ptr(em)))
        em = em.reshape(len(s), k + 1)
        return na, nt, [em[b, :na[b] + 1].tolist() for b in range(len(s))]

    def verify_step_sampled(self, draft, temperature: float, u_accept, u_sample: float, seq: int = 0):
        """The step with sampling: u_accept [k] and u_sample in [0, 1).  Returns (n_accepted, next_token, emitted list)."""
        na, nt, em = self.verify_step_sampled_batch([seq], [list(draft)], [temperature], [list(u_accept)], [u_sample])
        return int(na[0]), int(nt[0]), em[0]

    def verify_step_sampled_batch(self, seqs, drafts, temperature, u_accept, u_sample):
        """drafts, u_accept: [n_seqs, k]; temperature, u_sample: [n_seqs].  Returns (n_accepted[n_seqs], next_token[n_seqs], emitted[n_seqs][...])."""
        def f32(a, n, name):
            a = np.ascontiguousarray(np.asarray(a, dtype=np.float32).reshape(-1))
            if len(a) != n:
                _refuse(f"verify_step_sampled: {name} has {len(a)} entries, wanted {n}")
            return a
        s = _i32(seqs)
        d = np.asarray(drafts, dtype=np.int32).reshape(len(s), -1)
        k = d.shape[1]
        d = _i32(d)
        t, ua, us = f32(temperature, len(s), "temperature"), f32(u_accept, len(s) * k, "u_accept"), f32(u_sample, len(s), "u_sample")
        na, nt = np.zeros(len(s), np.int32), np.zeros(len(s), np.int32)
        em = np.zeros(len(s) * (k + 1), np.int32)
        fp = lambda a: a.ctypes.data_as(POINTER(c_float))
        self._ck(self.lib.llma_verify_step_sampled_batch(self._h, len(s), _ptr(s), _ptr(d), k, fp(t), fp(ua), fp(us), _ptr(na), _ptr(nt), _ptr(em)))
        em = em.reshape(len(s), k + 1)
        return na, nt, [em[b, :na[b] + 1].tolist() for b in range(len(s))]

    def generate(self, prompt, ref, doc_offsets, n: int, k: int, max_new: int, seq: int = 0):
        """Returns (tokens int32[max_new], trace list of (rows_in, emitted, doc, pos))."""
        p = _i32(prompt)
        r = _i32(ref if ref is not None else [])
        offs = _i32(doc_offsets if doc_offsets is not None else [0])
        out = np.zeros(max_new, np.int32)
        n_out, n_steps = c_int32(), c_int32()
        tr = (StepRec * max_new)()
        self._ck(self.lib.llma_generate(self._h, seq, _ptr(p), len(p), _ptr(r), _ptr(offs), len(offs) - 1, n, k, max_new,
                                        _ptr(out), byref(n_out), tr, byref(n_steps)))
        trace = [(t.rows_in, t.emitted, t.doc, t.pos) for t in tr[:n_steps.value]]
        return out[:n_out.value], trace

    def generate_batch(self, prompts, refs, n: int, k: int, max_new: int, seqs=None):
        """One LLMA decoding per sequence, all sequences in the same steps.  prompts: list of id
        arrays; refs: list of (ref, doc_offsets) or None per sequence.  Returns a list of
        (tokens int32[max_new], trace) per sequence."""
        B = len(prompts)
        s = _i32(seqs if seqs is not None else list(range(B)))
        ps = [_i32(p) for p in prompts]
        poff = _i32(np.concatenate([[0], np.cumsum([len(p) for p in ps])]))
        pcat = _i32(np.concatenate(ps))
        rs, offs, nd = [], [], []
        for r in refs:
            if r is None:
                rs.append(np.zeros(0, np.int32)); offs.append(np.zeros(1, np.int32)); nd.append(0)
            else:
                rs.append(_i32(r[0])); offs.append(_i32(r[1])); nd.append(len(offs[-1]) - 1)
        rcat, ocat, ndv = _i32(np.concatenate(rs)), _i32(np.concatenate(offs)), _i32(nd)
        out = np.zeros(B * max_new, np.int32)
        n_out, n_steps = np.zeros(B, np.int32), np.zeros(B, np.int32)
        tr = (StepRec * (B * max_new))()
        self._ck(self.lib.llma_generate_batch(self._h, B, _ptr(s), _ptr(pcat), _ptr(poff), _ptr(rcat), _ptr(ocat), _ptr(ndv),
                                              n, k, max_new, _ptr(out), _ptr(n_out), tr, _ptr(n_steps)))
        res = []
        for b in range(B):
            trace = [(t.rows_in, t.emitted, t.doc, t.pos) for t in tr[b * max_new:b * max_new + int(n_steps[b])]]
            res.append((out[b * max_new:b * max_new + int(n_out[b])].copy(), trace))
        return res

    # -- inspection
    def enable_logits_dump(self, rows: int):
        """Allocates a device buffer [rows, vocab] fp32 that every later forward fills."""
        self._dump = self._torch.zeros((rows, self.cfg.vocab), dtype=self._torch.float32, device=self.device)
        self._ck(self.lib.llma_set_logits_dump(self._h, c_void_p(self._dump.data_ptr()), rows))

    def disable_logits_dump(self):
        self._ck(self.lib.llma_set_logits_dump(self._h, None, 0))
        self._dump = None

    def logits(self, rows: int) -> np.ndarray:
        self._torch.cuda.synchronize(self.device)
        return self._dump[:rows].cpu().numpy()

    def set_option(self, option: int, value: int):
        self._ck(self.lib.llma_set_option(self._h, option, value))

    def kernel_timing(self):
        n, ms = c_int64(), c_double()
        self._ck(self.lib.llma_get_kernel_timing(self._h, byref(n), byref(ms)))
        return n.value, ms.value

    def time_ffn_gemm(self, rows: int, reps: int) -> float:
        us = c_double()
        self._ck(self.lib.llma_time_ffn_gemm(self._h, rows, reps, byref(us)))
        return us.value

    def time_step_gemm(self, which: int, rows: int, reps: int) -> float:
        us = c_double()
        self._ck(self.lib.llma_time_step_gemm(self._h, which, rows, reps, byref(us)))
        return us.value

    def describe(self) -> str:
        buf = ctypes.create_string_buffer(512)
        self._ck(self.lib.llma_describe(self._h, buf, 512))
        return buf.value.decode()

    def device_bytes(self) -> int:
        return int(self.lib.llma_device_bytes(self._h))
