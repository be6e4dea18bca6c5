// What the kernels over pages share (8-bit: kernels_paged.hip, 4-bit: kernels_paged_mx.hip): sums over a workgroup, rows as fp32, how a call's attention
// is cut into work, sequences and queries as the attention takes them, its outputs, and the join of parts.
#pragma once
#include "../../include/llma.h"
#include "paged.h"

// ---------------------------------------------------------------------------------------------
// sums over a workgroup
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ int wave_scan(int v) {              // inclusive, by register moves: a lane's group of 1, 2, 4 .. lanes and what lies before it
    const int lane = threadIdx.x & 63;
    int all = v;
    const auto step = [&](auto o) {
        const int other = lane_xor<o.value>(all);
        v += lane & o.value ? other : 0;
        all += other;
    };
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 8>{});
    step(std::integral_constant<int, 16>{});
    step(std::integral_constant<int, 32>{});
    return v;
}
// exclusive prefix sum of v over the workgroup's NW waves, *total the sum; part: LDS of at least NW words, free again after the next barrier
template <int NW>
__device__ __forceinline__ int block_scan(int v, int *part, int *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int in = wave_scan(v);
    __syncthreads();
    if (lane == 63) part[wave] = in;
    __syncthreads();
    int before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const int p = part[w];
        before += w < wave ? p : 0;
        sum += p;
    }
    *total = sum;
    return before + in - v;
}
// number of entries of the ascending list p[0 .. n) that are <= v
template <typename P>
__device__ __forceinline__ int count_le(const P *p, int n, int v) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p[mid] <= v) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// ---------------------------------------------------------------------------------------------
// rows of a call: eight neighbouring features as fp32
// ---------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
template <int TYPE>
__device__ __forceinline__ void row8(const void *p, int64_t at, float v[8]) {
    if constexpr (TYPE == ROWS_F32) {
        const f32x4 a = *(const f32x4 *)((const float *)p + at), b = *(const f32x4 *)((const float *)p + at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else if constexpr (TYPE == ROWS_F16) {
        const f16x8 a = *(const f16x8 *)((const _Float16 *)p + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
    } else {
        const u32x4 a = *(const u32x4 *)((const bf16_t *)p + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(a[e] << 16); v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u); }
    }
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// ---------------------------------------------------------------------------------------------
// attention: the work of a call
// ---------------------------------------------------------------------------------------------
#define ATTEND_CUS 256           // compute units; two workgroups each, one where three or four tiles fill the registers
#define ATTEND_MIN_PAGES 4       // of a share: a page per wave

#define ATTEND_WHOLE_PAGES 40    // whole sequences: of a table's row, at most
struct AttendPlan { int nt, tiles, shares; bool whole; };        // whole: sequences in place of shares
// row: bytes of K, and of V, that a position has per head; most_whole: pages of sequences that may stay whole
static AttendPlan attend_plan(int n_seqs, int max_blocks, int n_heads, int kv_heads, int row, int max_rows, int most_whole = ATTEND_WHOLE_PAGES) {
    const int64_t r = (int64_t)max_rows * (n_heads / kv_heads);
    AttendPlan p;
    p.nt = r <= 64 ? (int)((r + 15) / 16) : 4;
    p.tiles = (int)((r + 16 * p.nt - 1) / (16 * p.nt));
    const int64_t groups = (p.nt <= 2 ? 2 : 1) * ATTEND_CUS, columns = (int64_t)kv_heads * p.tiles;
    const int64_t pages = (int64_t)n_seqs * max_blocks, most = (pages + ATTEND_MIN_PAGES - 1) / ATTEND_MIN_PAGES;
    int64_t shares = groups / columns;
    if (shares > most) shares = most;
    p.shares = shares < 1 ? 1 : (int)shares;
    // pages beyond an equal share, at 16 KB of K and V each: 512 KB, or where whole sequences leave half of the compute units without work 256 KB and, of a
    // single one (which costs the least when cut), 192 KB
    const int64_t beyond = (max_blocks - pages * columns / groups) * row;
    p.whole = max_blocks <= most_whole && n_seqs * columns < 1 << 23 && beyond <= 128 * (n_seqs * columns >= ATTEND_CUS / 2 ? 32 : n_seqs > 1 ? 16 : 12);
    return p;
}
// work: [pages before every sequence, n_seqs + 1 ints, rounded up to 64][parts' O][parts' m][parts' l].  (Also where sequences stay whole: a workspace
// for some number of sequences does for fewer)
__host__ __device__ static inline int64_t attend_parts(const AttendPlan &p, int kv_heads) { return p.shares > 1 ? (int64_t)p.shares * 2 * kv_heads * p.tiles : 0; }
static inline int64_t attend_bytes(const AttendPlan &p, int n_seqs, int kv_heads, int dh) {
    return ((int64_t)(n_seqs + 1 + 63) / 64 * 64 + attend_parts(p, kv_heads) * 16 * p.nt * (dh + 2)) * 4;
}

struct AttendSeq { int slot, len, rows, row0, seen; };          // seen: the last position that its first row sees
// a sequence as the kernels take it: whatever the lists hold, nothing outside the buffers is reached
template <typename A>
__device__ __forceinline__ AttendSeq attend_seq(const A &a, int b) {
    AttendSeq s;
    s.row0 = a.row_offsets[b];
    s.rows = a.row_offsets[b + 1] - s.row0;
    const int all = s.rows;
    s.rows = s.rows > a.max_rows ? a.max_rows : s.rows;
    if (s.row0 < 0 || s.row0 > a.n_rows) s.rows = 0;
    else if (s.rows > a.n_rows - s.row0) s.rows = a.n_rows - s.row0;
    s.slot = a.slots ? a.slots[b] : b;
    s.len = a.lens[b];
    const int64_t most = (int64_t)a.max_blocks * PAGE_POS;
    if (s.len > most) s.len = (int)most;
    if (s.len < 0 || (unsigned)s.slot >= (unsigned)a.n_slots) s.len = 0;
    s.seen = s.rows > 0 ? s.len - all : 0;
    return s;
}
// (of one sequence for the whole wave: values that came through vector loads or LDS, into scalar registers)
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ AttendSeq uniform(AttendSeq s) { return AttendSeq{uniform(s.slot), uniform(s.len), uniform(s.rows), uniform(s.row0), uniform(s.seen)}; }
__device__ __forceinline__ int attend_pages(const AttendSeq &s) {      // a sequence without positions still has rows to write
    if (s.rows <= 0) return 0;
    return s.len < 1 ? 1 : (s.len + PAGE_POS - 1) / PAGE_POS;
}

// q: 16-byte operand pieces in LDS, [plane][tile][64-dim group][half][lane].  A thread's pieces on their way there: eight values each
template <int DH, int NT> constexpr int attend_pieces = NT * (DH / 64) * 2 * 64;
template <int DH, int NT> struct AttendQ { u32x4 raw[(attend_pieces<DH, NT> + 255) / 256][2]; };
// (KB: eight-feature steps of a lane that lie together: the 8-bit cache's lanes hold 16 features of every 64, the 4-bit one's dh / 4 in a row)
template <int DH, int NT, int TYPE, int KB = 2, typename A>
__device__ __forceinline__ void attend_load_q(const A &a, const AttendSeq &s, int head, int group, int r0, AttendQ<DH, NT> &q) {
#pragma unroll
    for (int u = 0; u < (attend_pieces<DH, NT> + 255) / 256; ++u) {
        const int i = u * 256 + threadIdx.x, lane = i & 63, step = (i >> 6) % (DH / 32), nt = (i >> 6) / (DH / 32);
        const int r = r0 + nt * 16 + (lane & 15), d = 32 * KB * (step / KB) + 8 * KB * (lane >> 4) + 8 * (step % KB);
        q.raw[u][0] = q.raw[u][1] = (u32x4){0, 0, 0, 0};
        if (i >= attend_pieces<DH, NT> || r >= s.rows * group) continue;
        const int row = s.row0 + r / group, h = head * group + r % group;
        if constexpr (TYPE == ROWS_TILED) {
            const size_t at = xtile_off(row, h * DH + d, a.tile_ksp, a.quads);
            q.raw[u][0] = *(const u32x4 *)((const bf16_t *)a.q + at);
            q.raw[u][1] = *(const u32x4 *)((const bf16_t *)a.q_lo + at);
        } else {
            const int64_t at = (int64_t)row * a.q_row + h * a.q_head + d;
            if constexpr (TYPE == ROWS_F32) {
                q.raw[u][0] = *(const u32x4 *)((const float *)a.q + at);
                q.raw[u][1] = *(const u32x4 *)((const float *)a.q + at + 4);
            } else {
                q.raw[u][0] = *(const u32x4 *)((const bf16_t *)a.q + at);
            }
        }
    }
}
template <int DH, int NT, int NQ, int TYPE>
__device__ __forceinline__ void attend_put_q(const AttendQ<DH, NT> &q, u32x4 *lds) {
    constexpr int PIECES = attend_pieces<DH, NT>;
#pragma unroll
    for (int u = 0; u < (PIECES + 255) / 256; ++u) {
        const int i = u * 256 + threadIdx.x;
        if (i >= PIECES) continue;
        if constexpr (TYPE == ROWS_BF16) {
            lds[i] = q.raw[u][0];
        } else if constexpr (TYPE == ROWS_TILED) {
            lds[i] = q.raw[u][0];
            lds[PIECES + i] = q.raw[u][1];
        } else {
            float v[8];
            if constexpr (TYPE == ROWS_F32) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(q.raw[u][e / 4][e % 4]);
            } else {
                const f16x8 h = __builtin_bit_cast(f16x8, q.raw[u][0]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                u32x4 p;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    p[w] = bf16_pair(v[2 * w], v[2 * w + 1]);
                    v[2 * w] -= __uint_as_float(p[w] << 16);
                    v[2 * w + 1] -= __uint_as_float(p[w] & 0xffff0000u);
                }
                lds[n * PIECES + i] = p;
            }
        }
    }
}
__device__ __forceinline__ f32x4 mfma16x16x32_half(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
}
__device__ __forceinline__ f32x4 times_pow2(f32x4 v, int e) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = __builtin_amdgcn_ldexpf(v[r], e);
    return v;
}
// a word's first n bytes (all for n >= 4, none for n <= 0)
__device__ __forceinline__ uint32_t bytes_below(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : ~(~0u << (8 * n)); }

template <int TYPE, typename A>
__device__ __forceinline__ void attend_store(const A &a, int row, int h, int d, f32x4 v) {      // four neighbouring features
    if constexpr (TYPE == ROWS_TILED) {
        const size_t at = xtile_off(row, h * a.c.dh + d, a.tile_out_ksp, a.quads);
        const float f[4] = {v[0], v[1], v[2], v[3]};
        u32x2 hi, lo;
        split4(f, hi, lo);
        *(u32x2 *)((bf16_t *)a.out + at) = hi;
        *(u32x2 *)((bf16_t *)a.out_lo + at) = lo;
    } else {
        const int64_t at = (int64_t)row * a.out_row + h * a.out_head + d;
        if constexpr (TYPE == ROWS_F32) {
            *(f32x4 *)((float *)a.out + at) = v;
        } else if constexpr (TYPE == ROWS_F16) {
            typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
            *(f16x4 *)((_Float16 *)a.out + at) = (f16x4){(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
        } else {
            *(u32x2 *)((bf16_t *)a.out + at) = (u32x2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        }
    }
}
// Planes of bf16 that hold a row type's q exactly (fp32: 24 bits), and a probability so that its rounding is lost in the output's: two leave 2^-16 of it, three
// 2^-24.  bf16 rows take one plane of fp16 (2^-11; the largest as 2^15, what lies 2^32 and more below it is lost) where the products are what bounds the call:
// from three tiles on, and for many rows.  us, two bf16 planes and one of fp16: two sequences of up to 2047 rows 332 and 272, 16 x 4096 with 33 rows of 32 heads 106 and 97, one of
// 512 rows over 1000 positions 39 and 34; up to two tiles nothing.  One plane of bf16 would be off by 2^-8, as an output's rounding is: 268, 98 and 35 us, and outputs 0.0022
// (rms, relative to 64 bits) off where 0.0017 is their own rounding.
template <int TYPE> constexpr int attend_nq = TYPE == ROWS_BF16 ? 1 : TYPE == ROWS_F32 ? 3 : 2;
template <int TYPE, bool HALF> constexpr int attend_np = HALF ? 1 : TYPE == ROWS_F32 ? 3 : 2;

// a share's part of one sequence: pages first .. last - 1 of it (none: last = 0)
struct AttendSeg { AttendSeq s; int b, first, last, pages; };
// a wave per row of a sequence that lies in several shares
template <int DH, int TYPE, typename A>
__global__ __launch_bounds__(256) void attend_join_kernel(A a, AttendPlan plan) {
    const int lane = threadIdx.x & 63, group = a.n_heads / a.c.heads;
    const int b = blockIdx.z, head = blockIdx.y, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int *const starts = (const int *)a.work;
    const int total = starts[a.n_seqs], p0 = starts[b], p1 = starts[b + 1];
    const AttendSeq s = attend_seq(a, b);
    if (r >= s.rows * group || p0 >= p1) return;
    int per = (total + plan.shares - 1) / plan.shares;
    per = per < ATTEND_MIN_PAGES ? ATTEND_MIN_PAGES : per;
    const int s0 = p0 / per, s1 = (p1 - 1) / per;
    if (s0 == s1) return;
    const int nt16 = 16 * plan.nt, tile = r / nt16, at16 = r % nt16;
    const int64_t parts = attend_parts(plan, a.c.heads);
    const float *const po = (const float *)a.work + (a.n_seqs + 1 + 63) / 64 * 64, *const pm = po + parts * nt16 * DH, *const pl = pm + parts * nt16;
    const auto place = [&](int sh) { return ((((int64_t)sh * 2 + (sh == s0)) * a.c.heads + head) * plan.tiles + tile) * nt16 + at16; };
    float m = LLMA_NEG_INF;
    for (int sh = s0 + lane; sh <= s1; sh += 64) m = fmaxf(m, pm[place(sh)]);
    butterfly<32>([&](auto o) { m = fmaxf(m, lane_xor<o.value>(m)); });
    const float ref = m == LLMA_NEG_INF ? 0.f : m;
    const int d = lane % (DH / 4) * 4, g0 = lane / (DH / 4);     // four features a lane; the wave's groups take parts in turn
    constexpr int GROUPS = 256 / DH;
    float l = 0.f;
    f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int sh = s0 + g0; sh <= s1; sh += GROUPS) {
        const int64_t at = place(sh);
        const float f = __builtin_amdgcn_exp2f(pm[at] - ref);
        l += pl[at] * f;
        o += *(const f32x4 *)(po + at * DH + d) * f;
    }
    const auto add = [&](auto off) {
        l += lane_xor<off.value>(l);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += lane_xor<off.value>(o[e]);
    };
    add(std::integral_constant<int, 32>{});
    if constexpr (DH == 64) add(std::integral_constant<int, 16>{});
    if (g0 == 0) attend_store<TYPE>(a, s.row0 + r / group, head * group + r % group, d, o * (l == 0.f ? 0.f : 1.f / l));
}
