// Argument structs and launchers of the paged 8-bit cache (kernels_paged.hip) and of sampled verification (kernels_sampled.hip).
#pragma once
#include "common.h"

// (weak: the host side is also linked against stand-ins of the launchers that a context cannot do without; one without these refuses
// paged contexts and sampled steps)
#define OPTIONAL __attribute__((weak))

#define PAGE_POS 64              // positions of a page (LLMA_PAGE)

// ---- the paged cache ---------------------------------------------------------------------------
// One allocation per plane, in pages of 64 positions, one block per (page, key head):
//   k [n_pages][heads][64][dh]   v [n_pages][heads][dh][64]   e4m3 codes (OCP, no infinities)
//   k_scale, v_scale [n_pages][heads]: powers of two; a cached value is code * scale.
// V lies transposed, so that both are the row-major A operand of their product: a lane's 16 bytes are 16 dims of one position of K,
// 16 positions of one dim of V, and 64 lanes take a whole KiB.  A power of two costs a floating-point code no
// precision and makes the product code * scale exact in bf16, where the matrix instructions take it, in the conversion that
// widens the code (v_cvt_scalef32_pk_bf16_fp8); a scale that grows re-rounds earlier codes only below e4m3's normal range.
struct PagedCache {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int n_pages, heads, dh;
};
enum RowType { ROWS_BF16 = 0, ROWS_F16 = 1, ROWS_F32 = 2, ROWS_TILED = 3 /* a context's own planes */ };

struct MapArgs {
    const int *lens, *rows, *slots;      // [n_slots], [n_seqs], [n_seqs] or null
    int n_seqs, n_slots;
    int *table;                          // [n_slots][max_blocks]
    int max_blocks;
    int *owned, *free_pages, *n_free;    // [n_slots], [n_pages], [1]
    int n_pages;
    int *row_offsets, *lens_after;       // [n_seqs + 1], [n_seqs]
    int *slot_map, *row_pos;             // [max_rows] each
    int max_rows;
    int *status;
    const int *last_live;                // [n_seqs] or null: rows behind row last_live[b] of sequence b carry no token and are mapped nowhere
};
OPTIONAL void launch_map_pages(const MapArgs &a, hipStream_t st);
// a context's pass as the calls above take it: rows[b] and slots[b] from its segments, or m rows (one sequence with last_live: *last_live + 1) of each of batch_slots
OPTIONAL void launch_pass_rows(const PromptSeg *segs, const int *batch_slots, int n_seqs, int m, const int *last_live, int *rows, int *slots, hipStream_t st);

struct AppendArgs {
    PagedCache c;
    const void *k, *v;                   // rows; ROWS_TILED: one slot of a context's tiled cache, position = row
    int64_t k_row, k_head, v_row, v_head;   // strides in elements (ROWS_TILED: k_head, v_head only)
    const int *slot_map;
    int n_rows;
    int type;
};
OPTIONAL void launch_append_paged(const AppendArgs &a, hipStream_t st);

struct AttendArgs {
    PagedCache c;
    const void *q, *q_lo;                // rows (q_lo: ROWS_TILED's lo plane)
    void *out, *out_lo;
    int64_t q_row, q_head, out_row, out_head;
    int type, n_heads;
    int tile_ksp, tile_out_ksp; bool quads;   // ROWS_TILED
    const int *table, *slots, *lens, *row_offsets;
    int n_seqs, n_slots, max_blocks, n_rows, max_rows;
    float scale;
    void *work;
};
OPTIONAL int64_t attend_paged_bytes(int n_seqs, int max_blocks, int n_heads, int kv_heads, int dh, int max_rows);
OPTIONAL void launch_attend_paged(const AttendArgs &a, hipStream_t st);

struct SampledArgs {
    const void *logits;                  // [n_seqs * (k + 1)] rows of `vocab`, row_stride elements apart
    int64_t row_stride;
    int type, vocab, n_seqs, k;
    const int *drafts, *n_draft;         // [n_seqs][draft_stride]; n_draft null: k everywhere
    int draft_stride;
    const float *probs;                  // [n_seqs * k][vocab] or null
    const float *temperature;            // [n_seqs] or null: 1
    const float *u_accept, *u_sample;    // [n_seqs * k], [n_seqs]
    int *n_accepted, *next, *emitted;    // [n_seqs], [n_seqs], [n_seqs][emit_stride]
    int emit_stride;
    void *work;
};
#define SAMPLED_MAX_K 63                 // (a lane per row)
#define SAMPLED_MAX_VOCAB (1 << 24)      // (ids and pieces of a row in 32 bits, 8192 ranges of it in a grid's second dimension)
#define SAMPLED_MAX_ROWS (1 << 22)       // of a call
OPTIONAL int64_t verify_sampled_bytes(int n_seqs, int k, int vocab);
OPTIONAL void launch_verify_sampled(const SampledArgs &a, hipStream_t st);
// words of a sampled step's inputs from pinned host memory into the device's
OPTIONAL void launch_take_words(const int *pinned, int *dev, int words, hipStream_t st);
struct CommitArgs {                      // what a sampled step leaves in its context
    const int *n_accepted, *next, *emitted;
    int emit_stride;
    const int *batch_slots;
    int *T, *pending;                    // [max_batch]
    int *io_nacc, *io_next, *io_emit;    // pinned, as the host reads them
    int io_stride, n_seqs;
};
OPTIONAL void launch_commit_sampled(const CommitArgs &a, hipStream_t st);
