// The stateless calls of serving on pages and of sampling (include/llma.h): argument checks, then the launchers.
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

template <typename C>
static int check_cache(const C *c, const char *who) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return refuse(LLMA_E_INVAL, "%s: null cache pointer", who);
    if (c->head_dim != 64 && c->head_dim != 128) return refuse(LLMA_E_INVAL, "%s: head_dim %d is not 64 or 128", who, c->head_dim);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return refuse(LLMA_E_INVAL, "%s: need n_pages >= 1 and 1 <= n_kv_heads <= 1024", who);
    if (c->n_pages > 0x7fffffff / LLMA_PAGE) return refuse(LLMA_E_RANGE, "%s: %d pages pass 32-bit slots", who, c->n_pages);
    if (!aligned(c->k) || !aligned(c->v)) return refuse(LLMA_E_INVAL, "%s: the cache is not 16-byte aligned", who);
    return LLMA_OK;
}
static int check_cache(const llma_paged_mx_cache *c, const char *who) {
    if (int rc = check_cache<llma_paged_mx_cache>(c, who)) return rc;
    if (!aligned(c->k_scale) || !aligned(c->v_scale)) return refuse(LLMA_E_INVAL, "%s: the cache is not 16-byte aligned", who);
    return LLMA_OK;
}
static PagedCache taken(const llma_paged_cache *c) {
    return PagedCache{(uint8_t *)c->k, (uint8_t *)c->v, c->k_scale, c->v_scale, c->n_pages, c->n_kv_heads, c->head_dim};
}
static PagedMxCache taken(const llma_paged_mx_cache *c) {
    return PagedMxCache{(uint8_t *)c->k, (uint8_t *)c->v, (uint8_t *)c->k_scale, (uint8_t *)c->v_scale, c->n_pages, c->n_kv_heads, c->head_dim};
}
// whether no two of n_rows x n_heads rows of head_dim values overlap
static bool rows_apart(int n_rows, int n_heads, int head_dim, int64_t row, int64_t head) {
    const bool heads_inside = head >= head_dim && (n_rows == 1 || row >= (n_heads - 1) * head + head_dim);
    const bool rows_inside = row >= head_dim && (n_heads == 1 || head >= (n_rows - 1) * row + head_dim);
    return heads_inside || rows_inside || n_rows * (int64_t)n_heads == 1;
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

template <typename C, typename F>
static int append_call(const C *cache, const void *k, const void *v, int32_t dtype, int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride,
                       int64_t v_head_stride, const int32_t *slot_map, int32_t n_rows, const char *who, F launch) {
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
    launch(type);
    return enqueued(who);
}
extern "C" int llma_append_paged(const llma_paged_cache *cache, const void *k, const void *v, int32_t dtype, int64_t k_row_stride, int64_t k_head_stride,
                                 int64_t v_row_stride, int64_t v_head_stride, const int32_t *slot_map, int32_t n_rows, void *hip_stream) {
    return append_call(cache, k, v, dtype, k_row_stride, k_head_stride, v_row_stride, v_head_stride, slot_map, n_rows, "llma_append_paged", [&](int type) {
        launch_append_paged(AppendArgs{taken(cache), k, v, k_row_stride, k_head_stride, v_row_stride, v_head_stride, slot_map, n_rows, type}, (hipStream_t)hip_stream);
    });
}
extern "C" int llma_append_paged_mx(const llma_paged_mx_cache *cache, const void *k, const void *v, int32_t dtype, int64_t k_row_stride, int64_t k_head_stride,
                                    int64_t v_row_stride, int64_t v_head_stride, const int32_t *slot_map, int32_t n_rows, void *hip_stream) {
    return append_call(cache, k, v, dtype, k_row_stride, k_head_stride, v_row_stride, v_head_stride, slot_map, n_rows, "llma_append_paged_mx", [&](int type) {
        launch_append_paged_mx(AppendMxArgs{taken(cache), k, v, k_row_stride, k_head_stride, v_row_stride, v_head_stride, slot_map, n_rows, type}, (hipStream_t)hip_stream);
    });
}

// rows out of either cache
template <typename C, typename A>
static int read_call(const C *cache, const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *first, const int32_t *row_offsets,
                     int32_t n_seqs, int32_t n_rows, void *k, void *v, int32_t dtype, int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride,
                     int64_t v_head_stride, void *hip_stream, const char *who, A a) {
    if (int rc = check_cache(cache, who)) return rc;
    const int type = row_type(dtype);
    if (type < 0) return refuse(LLMA_E_INVAL, "%s: unknown dtype %d", who, dtype);
    if (n_seqs < 0 || n_rows < 0 || max_blocks < 1) return refuse(LLMA_E_INVAL, "%s: need n_seqs, n_rows >= 0 and max_blocks >= 1", who);
    if (n_seqs > LLMA_PAGED_MAX_SEQS) return refuse(LLMA_E_RANGE, "%s: %d sequences, at most %d", who, n_seqs, LLMA_PAGED_MAX_SEQS);
    if (max_blocks > 0x7fffffff / LLMA_PAGE || (int64_t)n_rows * cache->n_kv_heads > (int64_t)1 << 28)
        return refuse(LLMA_E_RANGE, "%s: %d pages a sequence, %d rows of %d heads in one call", who, max_blocks, n_rows, cache->n_kv_heads);
    if (n_seqs == 0 || n_rows == 0) return LLMA_OK;
    if (!table || !row_offsets || !k || !v) return refuse(LLMA_E_INVAL, "%s: null pointer", who);
    if (n_slots < 1 || (!slots && n_slots < n_seqs)) return refuse(LLMA_E_RANGE, "%s: %d sequences in %d slots", who, n_seqs, n_slots);
    const int64_t es = item(type);
    if (!aligned(k) || !aligned(v) || !stride_ok(k_row_stride, es) || !stride_ok(k_head_stride, es) || !stride_ok(v_row_stride, es) || !stride_ok(v_head_stride, es))
        return refuse(LLMA_E_INVAL, "%s: rows must be 16-byte aligned (pointers and strides)", who);
    if (k == v) return refuse(LLMA_E_INVAL, "%s: k is v", who);
    if (!rows_apart(n_rows, cache->n_kv_heads, cache->head_dim, k_row_stride, k_head_stride) || !rows_apart(n_rows, cache->n_kv_heads, cache->head_dim, v_row_stride, v_head_stride))
        return refuse(LLMA_E_INVAL, "%s: rows overlap", who);
    a.c = taken(cache);
    a.k = k; a.v = v; a.k_row = k_row_stride; a.k_head = k_head_stride; a.v_row = v_row_stride; a.v_head = v_head_stride; a.type = type;
    a.table = table; a.slots = slots; a.first = first; a.row_offsets = row_offsets; a.n_seqs = n_seqs; a.n_slots = n_slots; a.max_blocks = max_blocks; a.n_rows = n_rows;
    launch_read_paged(a, (hipStream_t)hip_stream);
    return enqueued(who);
}
extern "C" int llma_read_paged(const llma_paged_cache *cache, const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *first,
                               const int32_t *row_offsets, int32_t n_seqs, int32_t n_rows, void *k, void *v, int32_t dtype, int64_t k_row_stride,
                               int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride, void *hip_stream) {
    return read_call(cache, table, slots, n_slots, max_blocks, first, row_offsets, n_seqs, n_rows, k, v, dtype, k_row_stride, k_head_stride, v_row_stride, v_head_stride, hip_stream,
                     "llma_read_paged", ReadArgs<PagedCache>{});
}
extern "C" int llma_read_paged_mx(const llma_paged_mx_cache *cache, const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *first,
                                  const int32_t *row_offsets, int32_t n_seqs, int32_t n_rows, void *k, void *v, int32_t dtype, int64_t k_row_stride,
                                  int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride, void *hip_stream) {
    return read_call(cache, table, slots, n_slots, max_blocks, first, row_offsets, n_seqs, n_rows, k, v, dtype, k_row_stride, k_head_stride, v_row_stride, v_head_stride, hip_stream,
                     "llma_read_paged_mx", ReadArgs<PagedMxCache>{});
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
template <typename C, typename A, typename B, typename F>
static int attend_call(const C *cache, const void *q, int32_t dtype, int32_t n_heads, int64_t q_row_stride, int64_t q_head_stride,
                       const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *lens, const int32_t *row_offsets, int32_t n_seqs,
                       int32_t n_rows, int32_t max_rows, float scale, void *out, int64_t out_row_stride, int64_t out_head_stride, void *work, int64_t work_bytes, const char *who, A a, B bytes, F launch) {
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
    if (scale != scale) return refuse(LLMA_E_INVAL, "%s: scale is NaN", who);
    // (rows of q may lie on top of each other, rows of out may not)
    if (!rows_apart(n_rows, n_heads, cache->head_dim, out_row_stride, out_head_stride)) return refuse(LLMA_E_INVAL, "%s: rows of out overlap", who);
    const int64_t need = bytes(n_seqs, max_blocks, n_heads, cache->n_kv_heads, cache->head_dim, max_rows);
    if (!aligned(work) || work_bytes < need) return refuse(LLMA_E_INVAL, "%s: needs a 16-byte aligned workspace of %lld bytes", who, (long long)need);
    a.c = taken(cache);
    a.q = q; a.out = out; a.q_row = q_row_stride; a.q_head = q_head_stride; a.out_row = out_row_stride; a.out_head = out_head_stride;
    a.type = type; a.n_heads = n_heads; a.table = table; a.slots = slots; a.lens = lens; a.row_offsets = row_offsets;
    a.n_seqs = n_seqs; a.n_slots = n_slots; a.max_blocks = max_blocks; a.n_rows = n_rows; a.max_rows = max_rows; a.scale = scale; a.work = work;
    launch(a);
    return enqueued(who);
}
extern "C" int llma_attend_paged(const llma_paged_cache *cache, const void *q, int32_t dtype, int32_t n_heads, int64_t q_row_stride, int64_t q_head_stride,
                                 const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *lens, const int32_t *row_offsets, int32_t n_seqs,
                                 int32_t n_rows, int32_t max_rows, float scale, void *out, int64_t out_row_stride, int64_t out_head_stride, void *work, int64_t work_bytes, void *hip_stream) {
    return attend_call(cache, q, dtype, n_heads, q_row_stride, q_head_stride, table, slots, n_slots, max_blocks, lens, row_offsets, n_seqs, n_rows, max_rows, scale, out, out_row_stride,
                       out_head_stride, work, work_bytes, "llma_attend_paged", AttendArgs{}, attend_paged_bytes,
                       [&](const AttendArgs &a) { launch_attend_paged(a, (hipStream_t)hip_stream); });
}
extern "C" int64_t llma_attend_paged_mx_workspace(int32_t n_seqs, int32_t max_blocks, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows) {
    if (int rc = check_attend(n_seqs, max_blocks, n_heads, n_kv_heads, head_dim, max_rows, "llma_attend_paged_mx_workspace")) return rc;
    return attend_paged_mx_bytes(n_seqs, max_blocks, n_heads, n_kv_heads, head_dim, max_rows < 1 ? 1 : max_rows);
}
extern "C" int llma_attend_paged_mx(const llma_paged_mx_cache *cache, const void *q, int32_t dtype, int32_t n_heads, int64_t q_row_stride, int64_t q_head_stride,
                                    const int32_t *table, const int32_t *slots, int32_t n_slots, int32_t max_blocks, const int32_t *lens, const int32_t *row_offsets, int32_t n_seqs,
                                    int32_t n_rows, int32_t max_rows, float scale, void *out, int64_t out_row_stride, int64_t out_head_stride, void *work, int64_t work_bytes, void *hip_stream) {
    return attend_call(cache, q, dtype, n_heads, q_row_stride, q_head_stride, table, slots, n_slots, max_blocks, lens, row_offsets, n_seqs, n_rows, max_rows, scale, out, out_row_stride,
                       out_head_stride, work, work_bytes, "llma_attend_paged_mx", AttendMxArgs{}, attend_paged_mx_bytes,
                       [&](const AttendMxArgs &a) { launch_attend_paged_mx(a, (hipStream_t)hip_stream); });
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

static int check_logprobs(int n_rows, int vocab, int n_top, const char *who) {
    if (n_rows < 0 || vocab < 1 || n_top < 0) return refuse(LLMA_E_INVAL, "%s: need n_rows, n_top >= 0 and vocab >= 1", who);
    if (n_top > LLMA_LOGPROBS_MAX_TOP) return refuse(LLMA_E_RANGE, "%s: %d alternatives, at most %d", who, n_top, LLMA_LOGPROBS_MAX_TOP);
    if (vocab > SAMPLED_MAX_VOCAB || n_rows > SAMPLED_MAX_ROWS || (int64_t)n_rows * vocab > (int64_t)1 << 40) return refuse(LLMA_E_RANGE, "%s: vocab %d, %d rows (at most 2^24, 2^22, together 2^40)", who, vocab, n_rows);
    return LLMA_OK;
}
extern "C" int64_t llma_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top) {
    if (int rc = check_logprobs(n_rows, vocab, n_top, "llma_token_logprobs_workspace")) return rc;
    return token_logprobs_bytes(n_rows, vocab, n_top);
}
extern "C" int llma_token_logprobs(const void *logits, int32_t dtype, int64_t row_stride, int32_t vocab, int32_t n_rows, const int32_t *tokens, const float *temperature,
                                   int32_t n_top, float *logprob, int32_t *rank, float *entropy, int32_t *top_tokens, float *top_logprobs, void *work, int64_t work_bytes,
                                   void *hip_stream) {
    const char *const who = "llma_token_logprobs";
    if (int rc = check_logprobs(n_rows, vocab, n_top, who)) return rc;
    const int type = row_type(dtype);
    if (type < 0) return refuse(LLMA_E_INVAL, "%s: unknown dtype %d", who, dtype);
    if (n_rows == 0) return LLMA_OK;
    if (!logits || !work || ((logprob || rank) && !tokens) || (n_top > 0 && (!top_tokens || !top_logprobs))) return refuse(LLMA_E_INVAL, "%s: null pointer", who);
    if (row_stride < vocab || row_stride > (int64_t)1 << 40 || (uintptr_t)logits % item(type)) return refuse(LLMA_E_INVAL, "%s: rows of %d logits %lld apart", who, vocab, (long long)row_stride);
    const int64_t need = token_logprobs_bytes(n_rows, vocab, n_top);
    if (!aligned(work) || work_bytes < need) return refuse(LLMA_E_INVAL, "%s: needs a 16-byte aligned workspace of %lld bytes", who, (long long)need);
    LogprobArgs a{};
    a.logits = logits; a.row_stride = row_stride; a.type = type; a.vocab = vocab; a.n_rows = n_rows; a.n_top = n_top; a.tokens = tokens; a.temperature = temperature;
    a.logprob = logprob; a.rank = rank; a.entropy = entropy; a.top_tokens = top_tokens; a.top_logprobs = top_logprobs; a.work = work;
    launch_token_logprobs(a, (hipStream_t)hip_stream);
    return enqueued(who);
}
