// The stateless calls of serving on pages (include/llma.h): argument checks, then the launchers.
#include <stdarg.h>
#include <stdio.h>

#include "../../include/llma.h"
#include "paged.h"

void llma_set_error_text(const char *text);     // llma_api.hip: text for llma_last_error(NULL)

static int refuse(int code, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    llma_set_error_text(buf);
    return code;
}
static int enqueued(const char *who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LLMA_OK : refuse(LLMA_E_HIP, "%s: %s", who, hipGetErrorString(e));
}
static bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }
static int row_type(int dtype) { return dtype == LLMA_DTYPE_BF16 ? ROWS_BF16 : dtype == LLMA_DTYPE_F16 ? ROWS_F16 : dtype == LLMA_DTYPE_F32 ? ROWS_F32 : -1; }
static int64_t item(int type) { return type == ROWS_F32 ? 4 : 2; }
static bool stride_ok(int64_t s, int64_t size) { return s >= 0 && s * size % 16 == 0 && s < (int64_t)1 << 40; }

static int check_cache(const llma_paged_cache *c, const char *who) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return refuse(LLMA_E_INVAL, "%s: null cache pointer", who);
    if (c->head_dim != 64 && c->head_dim != 128) return refuse(LLMA_E_INVAL, "%s: head_dim %d is not 64 or 128", who, c->head_dim);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return refuse(LLMA_E_INVAL, "%s: need n_pages >= 1 and 1 <= n_kv_heads <= 1024", who);
    if (c->n_pages > 0x7fffffff / LLMA_PAGE) return refuse(LLMA_E_RANGE, "%s: %d pages pass 32-bit slots", who, c->n_pages);
    if (!aligned(c->k) || !aligned(c->v)) return refuse(LLMA_E_INVAL, "%s: the cache is not 16-byte aligned", who);
    return LLMA_OK;
}
static PagedCache taken(const llma_paged_cache *c) {
    return PagedCache{(uint8_t *)c->k, (uint8_t *)c->v, c->k_scale, c->v_scale, c->n_pages, c->n_kv_heads, c->head_dim};
}

extern "C" int llma_map_pages(const int32_t *lens, const int32_t *rows, const int32_t *slots, int32_t n_seqs, int32_t n_slots, int32_t *table,
                              int32_t max_blocks, int32_t *owned, int32_t *free_pages, int32_t *n_free, int32_t n_pages, int32_t *row_offsets,
                              int32_t *lens_after, int32_t *slot_map, int32_t *row_pos, int32_t max_rows, int32_t *status, void *hip_stream) {
    const char *const who = "llma_map_pages";
    if (!lens || !rows || !table || !owned || !free_pages || !n_free || !row_offsets || !lens_after || !status) return refuse(LLMA_E_INVAL, "%s: null pointer", who);
    if (n_seqs < 1 || n_slots < 1 || max_blocks < 1 || n_pages < 1 || max_rows < 0) return refuse(LLMA_E_INVAL, "%s: need n_seqs, n_slots, max_blocks, n_pages >= 1 and max_rows >= 0", who);
    if (max_rows > 0 && (!slot_map || !row_pos)) return refuse(LLMA_E_INVAL, "%s: null slot_map or row_pos with max_rows > 0", who);
    if (max_rows > 1 << 30) return refuse(LLMA_E_RANGE, "%s: max_rows %d, at most 2^30", who, max_rows);
    if (n_slots > 65536) return refuse(LLMA_E_RANGE, "%s: %d slots, at most 65536", who, n_slots);
    if (n_seqs > n_slots) return refuse(LLMA_E_RANGE, "%s: %d sequences in %d slots", who, n_seqs, n_slots);
    if (n_pages > 0x7fffffff / LLMA_PAGE || max_blocks > 0x7fffffff / LLMA_PAGE) return refuse(LLMA_E_RANGE, "%s: pages pass 32-bit slots", who);
    if (lens_after == lens) return refuse(LLMA_E_INVAL, "%s: lens_after is lens", who);
    launch_map_pages(MapArgs{lens, rows, slots, n_seqs, n_slots, table, max_blocks, owned, free_pages, n_free, n_pages, row_offsets, lens_after, slot_map, row_pos, max_rows, status},
                     (hipStream_t)hip_stream);
    return enqueued(who);
}

extern "C" int llma_append_paged(const llma_paged_cache *cache, const void *k, const void *v, int32_t dtype, int64_t k_row_stride, int64_t k_head_stride,
                                 int64_t v_row_stride, int64_t v_head_stride, const int32_t *slot_map, int32_t n_rows, void *hip_stream) {
    const char *const who = "llma_append_paged";
    if (int rc = check_cache(cache, who)) return rc;
    const int type = row_type(dtype);
    if (type < 0) return refuse(LLMA_E_INVAL, "%s: unknown dtype %d", who, dtype);
    if (n_rows < 0) return refuse(LLMA_E_INVAL, "%s: n_rows %d", who, n_rows);
    if (n_rows == 0) return LLMA_OK;
    if (!k || !v || !slot_map) return refuse(LLMA_E_INVAL, "%s: null pointer", who);
    const int64_t es = item(type);
    if (!aligned(k) || !aligned(v) || !stride_ok(k_row_stride, es) || !stride_ok(k_head_stride, es) || !stride_ok(v_row_stride, es) || !stride_ok(v_head_stride, es))
        return refuse(LLMA_E_INVAL, "%s: rows must be 16-byte aligned (pointers and strides)", who);
    if ((int64_t)n_rows * cache->n_kv_heads > (int64_t)1 << 28) return refuse(LLMA_E_RANGE, "%s: %d rows of %d heads in one call", who, n_rows, cache->n_kv_heads);
    launch_append_paged(AppendArgs{taken(cache), k, v, k_row_stride, k_head_stride, v_row_stride, v_head_stride, slot_map, n_rows, type}, (hipStream_t)hip_stream);
    return enqueued(who);
}

// shapes that the attention's grids hold
static int check_attend(int n_seqs, int max_blocks, int n_heads, int kv_heads, int head_dim, int max_rows, const char *who) {
    if (n_seqs < 0 || max_rows < 0 || max_blocks < 1) return refuse(LLMA_E_INVAL, "%s: need n_seqs, max_rows >= 0 and max_blocks >= 1", who);
    if (n_seqs > LLMA_PAGED_MAX_SEQS) return refuse(LLMA_E_RANGE, "%s: %d sequences, at most %d", who, n_seqs, LLMA_PAGED_MAX_SEQS);
    if (kv_heads < 1 || kv_heads > 1024 || n_heads < 1 || n_heads % kv_heads) return refuse(LLMA_E_INVAL, "%s: %d query heads for %d key heads", who, n_heads, kv_heads);
    if (head_dim != 64 && head_dim != 128) return refuse(LLMA_E_INVAL, "%s: head_dim %d is not 64 or 128", who, head_dim);
    // positions of the whole batch, and a key head's query rows, are counted in 32 bits
    if ((int64_t)max_blocks * (n_seqs > 0 ? n_seqs : 1) > 0x7fffffff / LLMA_PAGE || (int64_t)max_rows * n_heads > (int64_t)1 << 26)
        return refuse(LLMA_E_RANGE, "%s: %d sequences x %d pages, %d rows x %d heads in one call", who, n_seqs, max_blocks, max_rows, n_heads);
    return LLMA_OK;
}
extern "C" int64_t llma_attend_paged_workspace(int32_t n_seqs, int32_t max_blocks, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows) {
    if (int rc = check_attend(n_seqs, max_blocks, n_heads, n_kv_heads, head_dim, max_rows, "llma_attend_paged_workspace")) return rc;
    return attend_paged_bytes(n_seqs, max_blocks, n_heads, n_kv_heads, head_dim, max_rows < 1 ? 1 : max_rows);
}
extern "C" int llma_attend_paged(const llma_paged_cache *cache, const void *q, int32_t dtype, int32_t n_heads, int64_t q_row_stride, int64_t q_head_stride,
                                 const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *lens,
                                 const int32_t *row_offsets, int32_t n_seqs, int32_t n_rows, int32_t max_rows, float scale, void *out, int64_t out_row_stride,
                                 int64_t out_head_stride, void *work, int64_t work_bytes, void *hip_stream) {
    const char *const who = "llma_attend_paged";
    if (int rc = check_cache(cache, who)) return rc;
    const int type = row_type(dtype);
    if (type < 0) return refuse(LLMA_E_INVAL, "%s: unknown dtype %d", who, dtype);
    if (int rc = check_attend(n_seqs, max_blocks, n_heads, cache->n_kv_heads, cache->head_dim, max_rows, who)) return rc;
    if (n_rows < 0) return refuse(LLMA_E_INVAL, "%s: n_rows %d", who, n_rows);
    if (n_seqs == 0 || n_rows == 0 || max_rows == 0) return LLMA_OK;
    if (!q || !out || !table || !lens || !row_offsets || !work) return refuse(LLMA_E_INVAL, "%s: null pointer", who);
    if (n_slots < 1 || (!slots && n_slots < n_seqs)) return refuse(LLMA_E_RANGE, "%s: %d sequences in %d slots", who, n_seqs, n_slots);
    const int64_t es = item(type);
    if (!aligned(q) || !aligned(out) || !stride_ok(q_row_stride, es) || !stride_ok(q_head_stride, es) || !stride_ok(out_row_stride, es) || !stride_ok(out_head_stride, es))
        return refuse(LLMA_E_INVAL, "%s: rows must be 16-byte aligned (pointers and strides)", who);
    if (out == q) return refuse(LLMA_E_INVAL, "%s: out is q", who);
    // (rows of q may lie on top of each other, rows of out may not)
    const bool heads_inside = out_head_stride >= cache->head_dim && (n_rows == 1 || out_row_stride >= (n_heads - 1) * out_head_stride + cache->head_dim);
    const bool rows_inside = out_row_stride >= cache->head_dim && (n_heads == 1 || out_head_stride >= (n_rows - 1) * out_row_stride + cache->head_dim);
    if (!(heads_inside || rows_inside || n_rows * (int64_t)n_heads == 1)) return refuse(LLMA_E_INVAL, "%s: rows of out overlap", who);
    const int64_t need = attend_paged_bytes(n_seqs, max_blocks, n_heads, cache->n_kv_heads, cache->head_dim, max_rows);
    if (!aligned(work) || work_bytes < need) return refuse(LLMA_E_INVAL, "%s: needs a 16-byte aligned workspace of %lld bytes", who, (long long)need);
    AttendArgs a{};
    a.c = taken(cache);
    a.q = q; a.out = out; a.q_row = q_row_stride; a.q_head = q_head_stride; a.out_row = out_row_stride; a.out_head = out_head_stride;
    a.type = type; a.n_heads = n_heads; a.table = table; a.slots = slots; a.lens = lens; a.row_offsets = row_offsets;
    a.n_seqs = n_seqs; a.n_slots = n_slots; a.max_blocks = max_blocks; a.n_rows = n_rows; a.max_rows = max_rows; a.scale = scale; a.work = work;
    launch_attend_paged(a, (hipStream_t)hip_stream);
    return enqueued(who);
}

static int check_sampled(int n_seqs, int k, int vocab, const char *who) {
    if (n_seqs < 0 || k < 0 || vocab < 1) return refuse(LLMA_E_INVAL, "%s: need n_seqs, k >= 0 and vocab >= 1", who);
    if (k > LLMA_SAMPLED_MAX_K) return refuse(LLMA_E_RANGE, "%s: k %d, at most %d", who, k, LLMA_SAMPLED_MAX_K);
    if (vocab > SAMPLED_MAX_VOCAB || (int64_t)n_seqs * (k + 1) > SAMPLED_MAX_ROWS) return refuse(LLMA_E_RANGE, "%s: vocab %d, %d sequences of %d rows (at most 2^24, 2^22 rows)", who, vocab, n_seqs, k + 1);
    return LLMA_OK;
}
extern "C" int64_t llma_verify_sampled_workspace(int32_t n_seqs, int32_t k, int32_t vocab) {
    if (int rc = check_sampled(n_seqs, k, vocab, "llma_verify_sampled_workspace")) return rc;
    return verify_sampled_bytes(n_seqs, k, vocab);
}
extern "C" int llma_verify_sampled(const void *logits, int32_t dtype, int64_t row_stride, int32_t vocab, int32_t n_seqs, int32_t k, const int32_t *drafts,
                                   const int32_t *n_draft, const float *draft_probs, const float *temperature, const float *u_accept, const float *u_sample,
                                   int32_t *n_accepted, int32_t *next_token, int32_t *emitted, void *work, int64_t work_bytes, void *hip_stream) {
    const char *const who = "llma_verify_sampled";
    if (int rc = check_sampled(n_seqs, k, vocab, who)) return rc;
    const int type = row_type(dtype);
    if (type < 0) return refuse(LLMA_E_INVAL, "%s: unknown dtype %d", who, dtype);
    if (n_seqs == 0) return LLMA_OK;
    if (!logits || !u_sample || !n_accepted || !next_token || !emitted || !work || (k > 0 && (!drafts || !u_accept))) return refuse(LLMA_E_INVAL, "%s: null pointer", who);
    if (row_stride < vocab || row_stride > (int64_t)1 << 40 || (uintptr_t)logits % item(type)) return refuse(LLMA_E_INVAL, "%s: rows of %d logits %lld apart", who, vocab, (long long)row_stride);
    const int64_t need = verify_sampled_bytes(n_seqs, k, vocab);
    if (!aligned(work) || work_bytes < need) return refuse(LLMA_E_INVAL, "%s: needs a 16-byte aligned workspace of %lld bytes", who, (long long)need);
    SampledArgs a{};
    a.logits = logits; a.row_stride = row_stride; a.type = type; a.vocab = vocab; a.n_seqs = n_seqs; a.k = k;
    a.drafts = drafts; a.draft_stride = k; a.n_draft = n_draft; a.probs = k > 0 ? draft_probs : nullptr; a.temperature = temperature; a.u_accept = u_accept; a.u_sample = u_sample;
    a.n_accepted = n_accepted; a.next = next_token; a.emitted = emitted; a.emit_stride = k + 1; a.work = work;
    launch_verify_sampled(a, (hipStream_t)hip_stream);
    return enqueued(who);
}
