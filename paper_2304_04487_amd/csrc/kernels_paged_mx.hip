// The paged 4-bit cache: the write into it, attention of a step's rows over it; and rows read back out of it and out of the 8-bit cache.
#include "paged_attend.h"

// ---------------------------------------------------------------------------------------------
// codes and scales
// ---------------------------------------------------------------------------------------------
// e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives.  The conversions read a scale's exponent bits alone (255: NaN), so one of four scale bytes
// gets into place by one shift, whatever its neighbours leave in the other bits.
template <int T> __device__ __forceinline__ float scale_byte(uint32_t w) { return __uint_as_float(T == 3 ? w >> 1 : w << (23 - 8 * T)); }
template <int T> __device__ __forceinline__ uint32_t widen2(uint32_t c, float scale) {       // byte T's two features as bf16
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, T));
}
// eight neighbouring features: an operand
__device__ __forceinline__ u32x4 widen8(uint32_t c, float scale) { return (u32x4){widen2<0>(c, scale), widen2<1>(c, scale), widen2<2>(c, scale), widen2<3>(c, scale)}; }
template <int T> __device__ __forceinline__ uint32_t widen2_half(uint32_t c, float scale) {  // as fp16
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, scale, T));
}
__device__ __forceinline__ u32x4 widen8_half(uint32_t c, float scale) { return (u32x4){widen2_half<0>(c, scale), widen2_half<1>(c, scale), widen2_half<2>(c, scale), widen2_half<3>(c, scale)}; }
__device__ __forceinline__ uint32_t nan_scales(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & w & 0x80808080u; }      // 0x80 in the bytes that are 255
// four words of four bytes, turned: word r gets byte r of each
__device__ __forceinline__ void turn4(uint32_t *w) {
    const uint32_t p = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), q = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
    const uint32_t t = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), u = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(q, p, 0x05040100u);
    w[1] = __builtin_amdgcn_perm(q, p, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(u, t, 0x05040100u);
    w[3] = __builtin_amdgcn_perm(u, t, 0x07060302u);
}
// exponent of the smallest power of two s from 2^-64 to 2^120 with amax / s <= 7: 6 is the largest code, and what lies up to 7 rounds to it by half a step as elsewhere
// (7 costs less than 6: 19.0 dB of normal values' blocks kept, 18.75 with 6, 18.8 with 8)
__device__ __forceinline__ int mx_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - 2 + ((b & 0x7fffffu) > 0x600000u);
    return e < -64 ? -64 : e > 120 ? 120 : e;
}

// ---------------------------------------------------------------------------------------------
// write into the cache
// ---------------------------------------------------------------------------------------------
// Per row, head and 32 features: s as above over the finite values, code = x / s rounded to nearest even (+-inf become +-6; a NaN makes the scale 255, the codes 0).
// 16 (8) lanes share a row's 128 (64) features, eight each.  A lane has the rows of up to four neighbouring positions, a quad, so that a byte of the
// transposed V leaves as one word for four positions, and so do the scales; a quad that is not whole leaves byte by byte.  A wave takes the quads that begin in its
// window of rows, 4 (8) at once: a prompt's rows are quads from its second page position divisible by four on, wherever it begins.
// Prompts are bound by memory: 4 of up to 2011 fp32 rows of 8 heads of 128, 58 MB, 13 us = 4.5 TB/s.  Steps by their chain of slots, rows and scale: 16 sequences of 9
// rows of 32 heads 6.2 us.
template <int DH, int TYPE, bool KEYS>
__device__ __forceinline__ void append_mx_quad(const AppendMxArgs &a, int head, int row, int n, int slot, int oct) {
    constexpr int FB = DH / 32;
    const int page = slot / PAGE_POS, at = slot % PAGE_POS;
    const size_t block = (size_t)page * a.c.heads + head;
    float v[4][8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = row + (r < n ? r : 0);
        if constexpr (KEYS) row8<TYPE>(a.k, i * a.k_row + head * a.k_head + 8 * oct, v[r]);
        else row8<TYPE>(a.v, i * a.v_row + head * a.v_head + 8 * oct, v[r]);
    }
    uint32_t codes[4], scales = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float amax = 0.f;
        int nan = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = fabsf(v[r][e]);
            amax = fmaxf(amax, x < __builtin_huge_valf() ? x : 0.f);
            nan |= x != x;
        }
        amax = fmaxf(amax, lane_xor<1>(amax));
        nan |= lane_xor<1>(nan);
        amax = fmaxf(amax, lane_xor<2>(amax));
        nan |= lane_xor<2>(nan);
        const int e = mx_exponent(amax);
        const float s = pow2(e);
        uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[r][0], v[r][1], s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[r][2], v[r][3], s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[r][4], v[r][5], s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[r][6], v[r][7], s, 3);
        codes[r] = nan ? 0u : c;
        scales |= (uint32_t)(nan ? 255 : e + 127) << 8 * r;
    }
    uint8_t *const sc = (KEYS ? a.c.k_scale : a.c.v_scale) + (block * FB + oct / 4) * PAGE_POS + at;
    const bool whole = n == 4;                                   // (then at is a multiple of four)
    if (oct % 4 == 0) {
        if (whole) *(uint32_t *)sc = scales;
        else
            for (int r = 0; r < n; ++r) sc[r] = (uint8_t)(scales >> 8 * r);
    }
    if constexpr (KEYS) {
        uint32_t *const to = (uint32_t *)(a.c.k + (block * PAGE_POS + at) * (DH / 2)) + oct;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < n) to[r * (DH / 8)] = codes[r];
    } else {
        uint8_t *const to = a.c.v + (block * (DH / 2) + 4 * oct) * PAGE_POS + at;
        if (whole) {
            turn4(codes);
#pragma unroll
            for (int j = 0; j < 4; ++j) *(uint32_t *)(to + j * PAGE_POS) = codes[j];
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[j * PAGE_POS + r] = (uint8_t)(codes[r] >> 8 * j);
        }
    }
}
#define APPEND_MX_WINDOW 16
template <int DH, int TYPE>
__global__ __launch_bounds__(256) void append_paged_mx_kernel(AppendMxArgs a, int n_windows) {
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int units = 2 * a.c.heads, unit = (int)(id % units);
    if (id / units >= n_windows) return;
    const int r0 = (int)(id / units) * APPEND_MX_WINDOW, head = unit >> 1;
    // lanes 0 .. 19: the window's slots, and those of three rows behind it; lane 63: the row's before it
    const int i = lane == 63 ? r0 - 1 : r0 + lane;
    int slot = -1;
    if ((lane < APPEND_MX_WINDOW + 3 || lane == 63) && i >= 0 && i < a.n_rows) slot = a.slot_map[i];
    if (slot < 0 || slot / PAGE_POS >= a.c.n_pages) slot = -1;
    const int before = __shfl(slot, (lane + 63) & 63);
    const bool follows = slot >= 0 && before >= 0 && slot == before + 1 && slot % 4 != 0;         // the row before it, in its quad
    const uint32_t on = (uint32_t)__ballot(follows && lane < 32);
    uint32_t starts = (uint32_t)__ballot(slot >= 0 && !follows && lane < APPEND_MX_WINDOW);
    constexpr int LANES = DH / 8, GROUPS = 64 / LANES;
    const int oct = lane % LANES, group = lane / LANES;
    while (starts) {
        int mine = -1;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            if (starts && g == group) mine = __builtin_ctz(starts);
            starts &= starts - 1;
        }
        const int from = mine < 0 ? 0 : mine, n = 1 + __builtin_ctz(~(on >> (from + 1)));         // (rows that follow: at most three, as a quad ends at a multiple of four)
        const int first = __shfl(slot, from);
        if (mine < 0) continue;
        if (unit & 1) append_mx_quad<DH, TYPE, false>(a, head, r0 + from, n, first, oct);
        else append_mx_quad<DH, TYPE, true>(a, head, r0 + from, n, first, oct);
    }
}
void launch_append_paged_mx(const AppendMxArgs &a, hipStream_t st) {
    if (a.n_rows < 1) return;
    const int n_windows = (a.n_rows + APPEND_MX_WINDOW - 1) / APPEND_MX_WINDOW;
    const int64_t blocks = ((int64_t)n_windows * 2 * a.c.heads + 3) / 4;
    auto of = [&](auto dh) {
        constexpr int DH = decltype(dh)::value;
        if (a.type == ROWS_BF16) hipLaunchKernelGGL((append_paged_mx_kernel<DH, ROWS_BF16>), dim3((unsigned)blocks), dim3(256), 0, st, a, n_windows);
        else if (a.type == ROWS_F16) hipLaunchKernelGGL((append_paged_mx_kernel<DH, ROWS_F16>), dim3((unsigned)blocks), dim3(256), 0, st, a, n_windows);
        else hipLaunchKernelGGL((append_paged_mx_kernel<DH, ROWS_F32>), dim3((unsigned)blocks), dim3(256), 0, st, a, n_windows);
    };
    if (a.c.dh == 128) of(std::integral_constant<int, 128>{});
    else of(std::integral_constant<int, 64>{});
}

// ---------------------------------------------------------------------------------------------
// rows out of the cache
// ---------------------------------------------------------------------------------------------
// Row j of sequence b is position first[b] + j.  A run = rows of one sequence inside one page; a workgroup takes one head of the runs that begin in its window of
// rows (64: a long sequence's one run).  A lane stores 16 bytes of a row, eight neighbouring lanes 128.  K's rows lie as they leave.  V's lie across: a lane takes four
// positions of its features, turns them in registers and has its features of four rows.
// Bound by memory, mostly by what is written: prefixes of five sequences of up to 4001 positions x 32 heads of 128 from 8 bits to bf16, 301 MB in 60 us = 5.0 TB/s; 37
// of up to 1900 x 8 heads from 4 bits to fp32, 400 MB, 90 us = 4.4 TB/s (118 with 32 bytes a lane in two halves, K and V one after the other).  Short ones by the chain
// of offsets, table and page: 1001 positions of 8 heads of 64 4.7 us, 16 sequences of 9 rows of 32 heads 5.3 (18.7 in windows of 64 rows).
struct ReadRun { int row, n, page, at; };                        // page -1: none, the rows become 0
template <int TYPE> constexpr int read_features = TYPE == ROWS_F32 ? 4 : 8;      // of 16 bytes
template <int TYPE>
__device__ __forceinline__ void store16(void *p, int64_t at, const float (&v)[read_features<TYPE>]) {
    if constexpr (TYPE == ROWS_F32) *(f32x4 *)((float *)p + at) = (f32x4){v[0], v[1], v[2], v[3]};
    else if constexpr (TYPE == ROWS_F16) *(u32x4 *)((bf16_t *)p + at) = (u32x4){half_pair(v[0], v[1]), half_pair(v[2], v[3]), half_pair(v[4], v[5]), half_pair(v[6], v[7])};
    else *(u32x4 *)((bf16_t *)p + at) = (u32x4){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
}
// four or eight neighbouring features' values
typedef __attribute__((ext_vector_type(2))) float f32x2;
template <bool MX, int F>
__device__ __forceinline__ void values_of(const uint32_t (&c)[2], float scale, float (&v)[F]) {
    if constexpr (MX) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], scale, 1);
        v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
        if constexpr (F == 8) {
            const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], scale, 3);
            v[4] = d[0]; v[5] = d[1]; v[6] = e[0]; v[7] = e[1];
        }
    } else {
#pragma unroll
        for (int w = 0; w < F / 4; ++w) {
            v[4 * w] = __builtin_amdgcn_cvt_f32_fp8((int)c[w], 0) * scale;
            v[4 * w + 1] = __builtin_amdgcn_cvt_f32_fp8((int)c[w], 1) * scale;
            v[4 * w + 2] = __builtin_amdgcn_cvt_f32_fp8((int)c[w], 2) * scale;
            v[4 * w + 3] = __builtin_amdgcn_cvt_f32_fp8((int)c[w], 3) * scale;
        }
    }
}
template <typename C, int DH, int TYPE>
__device__ __forceinline__ void read_run(const ReadArgs<C> &a, int head, const ReadRun &r) {
    constexpr bool MX = std::is_same_v<C, PagedMxCache>;
    constexpr int F = read_features<TYPE>, LANES = DH / F, ROWS = 256 / LANES, PASSES = PAGE_POS / ROWS;
    constexpr int WORDS = MX ? F / 2 : F, VPASSES = (LANES * (PAGE_POS / 4) + 255) / 256;      // WORDS: of four positions each
    const size_t block = (size_t)(r.page < 0 ? 0 : r.page) * a.c.heads + head;
    // ---- K's codes, then V's: all requested before the first is used
    const int k_at = threadIdx.x % LANES, j0 = threadIdx.x / LANES;
    uint32_t c[PASSES][2];
    float ks[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int j = j0 + p * ROWS, pos = r.at + (j < r.n ? j : 0);
        const uint8_t *const from = a.c.k + (block * PAGE_POS + pos) * (MX ? DH / 2 : DH) + k_at * (MX ? F / 2 : F);
        c[p][1] = 0;
        if constexpr (MX && F == 4) c[p][0] = *(const uint16_t *)from;
        else if constexpr (MX || F == 4) c[p][0] = *(const uint32_t *)from;
        else {
            const u32x2 w = *(const u32x2 *)from;
            c[p][0] = w[0];
            c[p][1] = w[1];
        }
        if constexpr (MX) ks[p] = __uint_as_float((uint32_t)a.c.k_scale[(block * (DH / 32) + k_at * F / 32) * PAGE_POS + pos] << 23);
        else ks[p] = a.c.k_scale[block];
    }
    uint32_t w[VPASSES][WORDS], sc[VPASSES];
#pragma unroll
    for (int p = 0; p < VPASSES; ++p) {
        const int t = 256 * p + threadIdx.x, at = t % 8 + t / (8 * 16) * 8, quad = t / 8 % 16;
        if (at >= LANES || 4 * quad + 3 < r.at || 4 * quad >= r.at + r.n) continue;
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[p][j] = *(const uint32_t *)(a.c.v + (block * (MX ? DH / 2 : DH) + WORDS * at + j) * PAGE_POS + 4 * quad);
        if constexpr (MX) sc[p] = *(const uint32_t *)(a.c.v_scale + (block * (DH / 32) + at * F / 32) * PAGE_POS + 4 * quad);
        else sc[p] = __float_as_uint(a.c.v_scale[block]);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int j = j0 + p * ROWS;
        if (j >= r.n) continue;
        float v[F];
        values_of<MX, F>(c[p], ks[p], v);
#pragma unroll
        for (int e = 0; e < F; ++e) v[e] = r.page < 0 ? 0.f : v[e];
        store16<TYPE>(a.k, (r.row + j) * a.k_row + head * a.k_head + F * k_at, v);
    }
#pragma unroll
    for (int p = 0; p < VPASSES; ++p) {
        const int t = 256 * p + threadIdx.x, at = t % 8 + t / (8 * 16) * 8, quad = t / 8 % 16;
        if (at >= LANES || 4 * quad + 3 < r.at || 4 * quad >= r.at + r.n) continue;
        uint32_t row[4][2];                                      // the codes of a row's features
        if constexpr (WORDS == 2) {
            const uint32_t x = __builtin_amdgcn_perm(w[p][1], w[p][0], 0x05010400u), y = __builtin_amdgcn_perm(w[p][1], w[p][0], 0x07030602u);
            row[0][0] = x;
            row[1][0] = x >> 16;
            row[2][0] = y;
            row[3][0] = y >> 16;
        } else {
#pragma unroll
            for (int g = 0; g < WORDS; g += 4) {
                turn4(w[p] + g);
#pragma unroll
                for (int j = 0; j < 4; ++j) row[j][g / 4] = w[p][g + j];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = 4 * quad + j - r.at;
            if (i < 0 || i >= r.n) continue;
            float v[F];
            values_of<MX, F>(row[j], __uint_as_float(MX ? (sc[p] >> 8 * j & 255u) << 23 : sc[p]), v);
#pragma unroll
            for (int e = 0; e < F; ++e) v[e] = r.page < 0 ? 0.f : v[e];
            store16<TYPE>(a.v, (r.row + i) * a.v_row + head * a.v_head + F * at, v);
        }
    }
}
template <typename C, int DH, int TYPE>
__global__ __launch_bounds__(256) void read_paged_kernel(ReadArgs<C> a, int window) {
    extern __shared__ int offsets[];                             // [n_seqs + 1]
    __shared__ ReadRun runs[64];
    __shared__ int n_runs;
    const int head = blockIdx.x % a.c.heads, r0 = blockIdx.x / a.c.heads * window;
    for (int b = threadIdx.x; b <= a.n_seqs; b += 256) offsets[b] = a.row_offsets[b];
    __syncthreads();
    if (threadIdx.x < 64) {
        const int i = r0 + threadIdx.x;
        ReadRun run{i, 0, -1, 0};
        bool begins = false;
        if ((int)threadIdx.x < window && i < a.n_rows && i >= offsets[0] && i < offsets[a.n_seqs]) {
            int b = count_le(offsets, a.n_seqs + 1, i) - 1;
            b = b < 0 ? 0 : b >= a.n_seqs ? a.n_seqs - 1 : b;
            const int64_t pos = (int64_t)(a.first ? a.first[b] : 0) + i - offsets[b];
            const int slot = a.slots ? a.slots[b] : b, in = (int)(pos & (PAGE_POS - 1));
            begins = i == offsets[b] || in == 0;
            if (begins) {
                run.at = in;
                const int64_t left = (int64_t)offsets[b + 1] - i, rest = a.n_rows - i;
                run.n = PAGE_POS - in;
                run.n = left < run.n ? (int)left : run.n;
                run.n = rest < run.n ? (int)rest : run.n;
                if (pos >= 0 && pos < (int64_t)a.max_blocks * PAGE_POS && (unsigned)slot < (unsigned)a.n_slots) run.page = a.table[(size_t)slot * a.max_blocks + pos / PAGE_POS];
                if ((unsigned)run.page >= (unsigned)a.c.n_pages) run.page = -1;
            }
        }
        const unsigned long long all = __ballot(begins);
        if (begins) runs[__popcll(all & ((1ull << threadIdx.x) - 1))] = run;
        if (threadIdx.x == 0) n_runs = __popcll(all);
    }
    __syncthreads();
    for (int k = 0; k < n_runs; ++k) read_run<C, DH, TYPE>(a, head, runs[k]);
}
template <typename C>
static void launch_read(const ReadArgs<C> &a, hipStream_t st) {
    if (a.n_seqs < 1 || a.n_rows < 1) return;
    // windows of a page's rows; where sequences have fewer, and there are too few windows for the chip, smaller ones: a workgroup takes its window's runs one after the other
    int window = 64;
    while (window > 4 && (int64_t)a.n_seqs * window > a.n_rows && (int64_t)((a.n_rows + window - 1) / window) * a.c.heads < 1024) window /= 2;
    const unsigned blocks = (unsigned)((a.n_rows + window - 1) / window * a.c.heads);
    const size_t bytes = (size_t)(a.n_seqs + 1) * 4;
    auto of = [&](auto dh) {
        constexpr int DH = decltype(dh)::value;
        if (a.type == ROWS_BF16) hipLaunchKernelGGL((read_paged_kernel<C, DH, ROWS_BF16>), dim3(blocks), dim3(256), bytes, st, a, window);
        else if (a.type == ROWS_F16) hipLaunchKernelGGL((read_paged_kernel<C, DH, ROWS_F16>), dim3(blocks), dim3(256), bytes, st, a, window);
        else hipLaunchKernelGGL((read_paged_kernel<C, DH, ROWS_F32>), dim3(blocks), dim3(256), bytes, st, a, window);
    };
    if (a.c.dh == 128) of(std::integral_constant<int, 128>{});
    else of(std::integral_constant<int, 64>{});
}
void launch_read_paged(const ReadArgs<PagedCache> &a, hipStream_t st) { launch_read(a, st); }
void launch_read_paged(const ReadArgs<PagedMxCache> &a, hipStream_t st) { launch_read(a, st); }

// ---------------------------------------------------------------------------------------------
// attention over the pages
// ---------------------------------------------------------------------------------------------
// The products, shares, whole sequences and the join are those of the 8-bit cache's kernel: S^T = K Q^T, O^T = V^T P^T, 16 rows a tile, one pass with the running maximum and
// sum of the softmax in fp32.  What differs is how a lane finds its operands:
//   K: row r of score tile t is position 4 r + t of the page, so that the four tiles' scales of a lane's block of 32 features are the bytes of one word, and
//   a lane's 16 probabilities those of 16 neighbouring positions, which its 16 bytes of V hold.  At head_dim 128 a lane has a block of 32 features (16 bytes), at 64 half of one.
//   V: a byte is two features of a position.  Widened (with its position's scale) it is a pair across features; two positions' pairs, exchanged by halves, are
//   pairs along the positions, of an even and of an odd feature: block jj of 32 features makes two operands, features 32 jj + 2 i and 32 jj + 2 i + 1.
// Both products see exactly what codes and scales stand for.
// Steps are bound by the read of the cache up to one tile of rows: 16 sequences of up to 4096 positions, 9 rows of 32 heads of 128, 192 MB in 36 us with the cache's
// bytes still in the last-level cache, 40 to 47 without = 4.1 to 4.8 TB/s (a kernel of the same mapping that only loads: 31.5 with).  From two tiles on by the products
// and the vector instructions beside them, which take turns rather than overlap: 61 of 5 rows, four query heads a key head, fp16, 358 MB in 95 us (load-only 74), a
// third of the cycles in matrix instructions, half in vector instructions.  Not faster: products in another order, a page's scores a page ahead of its other product
// (39 and 115 us), one word of scales a lane exchanged between lanes; one fp16 plane of probabilities spills here (47 us).
// Other matrix instructions would take the codes as they are, with their scales, beside queries in planes of 8 bits: their sums are off by 1e-5 of the largest product (rms).
// rare: a page's V has scales that stand for NaN where not all rows see them.  The rows that see one get it in its 32 features.  seen: 0x80 in the bytes of the lane's 16 positions
template <int DH, int NT>
__device__ __forceinline__ void attend_mx_nans(const u32x4 (&nans)[DH / 32], int base, const int (&limit)[NT], f32x4 (&o)[NT][DH / 16]) {
    const int kb = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int j = 0; j < DH / 32; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            int hit = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) hit |= (nans[j][w] & bytes_below(limit[n] + 1 - base - 16 * kb - 4 * w)) != 0;
            hit |= lane_xor<16>(hit);
            hit |= lane_xor<32>(hit);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                o[n][2 * j][r] = hit ? __builtin_nanf("") : o[n][2 * j][r];
                o[n][2 * j + 1][r] = hit ? __builtin_nanf("") : o[n][2 * j + 1][r];
            }
        }
}
// words i = 2 u, 2 u + 1 of a lane's 16 bytes of V: the operands of its even and its odd feature
__device__ __forceinline__ void widen_v(const u32x4 &c, const u32x4 &s, int u, u32x4 &even, u32x4 &odd) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = c[2 * u + h], b = s[2 * u + h];
        const uint32_t p0 = widen2<0>(w, scale_byte<0>(b)), p1 = widen2<1>(w, scale_byte<1>(b)), p2 = widen2<2>(w, scale_byte<2>(b)), p3 = widen2<3>(w, scale_byte<3>(b));
        even[2 * h] = __builtin_amdgcn_perm(p1, p0, 0x05040100u);
        odd[2 * h] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
        even[2 * h + 1] = __builtin_amdgcn_perm(p3, p2, 0x05040100u);
        odd[2 * h + 1] = __builtin_amdgcn_perm(p3, p2, 0x07060302u);
    }
}
// planes of the queries in LDS: attend_nq of bf16, and fp16 rows as they are
template <int TYPE> constexpr int attend_mx_planes = attend_nq<TYPE> + (TYPE == ROWS_F16);
template <int DH, int NT, int TYPE> constexpr int attend_mx_lds = 16 * (attend_mx_planes<TYPE> * attend_pieces<DH, NT> > 4 * NT * (DH / 16) * 64 ? attend_mx_planes<TYPE> * attend_pieces<DH, NT> : 4 * NT * (DH / 16) * 64);
// no byte outside 104 .. 139: a code times such a scale is exact in fp16
__device__ __forceinline__ bool half_scales(uint32_t w) {
    const uint32_t low = w & 0x7f7f7f7fu;
    return (((low + 0x18181818u) | w) & ~((low + 0x74747474u) & w) & 0x80808080u) == 0x80808080u;
}
#define ATTEND_KEPT 256          // sequences whose lengths and rows the workgroup keeps in LDS

template <int DH, int NT, int TYPE>
__global__ __launch_bounds__(256, NT <= 2 ? 2 : 1) void attend_paged_mx_kernel(AttendMxArgs a, AttendPlan plan) {
    constexpr int NQ = attend_nq<TYPE>, NP = attend_np<TYPE, false>;
    constexpr int STEPS = DH / 32, FB = DH / 32, DT = DH / 16, PIECES = attend_pieces<DH, NT>;     // STEPS: products a score takes, of 32 features
    typedef std::conditional_t<DH == 128, u32x4, u32x2> KBytes;                                     // a lane's DH / 4 features of a position
    extern __shared__ u32x4 lds[];
    u32x4 *const q = lds;
    f32x4 *const osum = (f32x4 *)lds;                            // the four waves' sums, in the queries' place once they are used
    __shared__ float ml[4][2][NT * 16];
    __shared__ int part[4];
    __shared__ AttendSeq kept[ATTEND_KEPT];
    int *const starts = (int *)((char *)lds + attend_mx_lds<DH, NT, TYPE>);         // [n_seqs + 1]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shares = plan.whole ? a.n_seqs : plan.shares, share = blockIdx.x % shares, head = blockIdx.x / shares % a.c.heads, tile = blockIdx.x / shares / a.c.heads;
    const int group = a.n_heads / a.c.heads, r0 = tile * NT * 16;
    // ---- where the sequences' pages begin
    const int n_seqs = plan.whole ? 1 : a.n_seqs;
    int total = 0;
    if (plan.whole) {
        const AttendSeq s = attend_seq(a, share);
        total = attend_pages(s);
        if (threadIdx.x == 0) {
            kept[0] = s;
            starts[0] = 0;
        }
    }
    for (int b0 = 0; b0 < a.n_seqs && !plan.whole; b0 += 256) {
        const int b = b0 + threadIdx.x;
        int sum, pages = 0;
        if (b < a.n_seqs) {
            const AttendSeq s = attend_seq(a, b);
            pages = attend_pages(s);
            if (b < ATTEND_KEPT) kept[b] = s;
        }
        const int at = block_scan<4>(pages, part, &sum);
        if (b < a.n_seqs) starts[b] = total + at;
        total += sum;
    }
    if (threadIdx.x == 0) starts[n_seqs] = total;
    __syncthreads();
    if (plan.shares > 1 && !plan.whole && blockIdx.x == 0)       // (for attend_join_kernel)
        for (int b = threadIdx.x; b <= a.n_seqs; b += 256) ((int *)a.work)[b] = starts[b];
    total = uniform(total);
    int per = plan.whole ? total : (total + plan.shares - 1) / plan.shares;
    per = per < ATTEND_MIN_PAGES ? ATTEND_MIN_PAGES : per;
    const int64_t from = plan.whole ? 0 : (int64_t)share * per;
    if (from >= total) return;
    const int p0 = (int)from, p1 = p0 + per < total ? p0 + per : total;
    // (not 0: minus infinity has to stay that.  A negative scale turns the queries' signs, so that the largest score is the largest product)
    const float by = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 1e-37f);
    const uint32_t turn = a.scale < 0.f ? TYPE == ROWS_F32 ? 0x80000000u : 0x80008000u : 0u;
    const int kb = lane >> 4, col = lane & 15;
    const uint32_t k_off = 4 * col * (DH / 2) + kb * (DH / 8), ks_off = (kb * FB / 4) * PAGE_POS + 4 * col, v_off = col * PAGE_POS + 16 * kb;

    // the share's part of sequence b, or of the next that has rows in this tile
    const auto segment = [&](int b) {
        AttendSeg g{};
        for (; b < n_seqs; ++b) {
            const int begin = uniform(starts[b]), end = uniform(starts[b + 1]);
            if (begin >= p1) break;
            const int first = p0 > begin ? p0 - begin : 0, last = (p1 < end ? p1 : end) - begin;
            if (first >= last) continue;
            const AttendSeq s = uniform(b < ATTEND_KEPT ? kept[b] : attend_seq(a, b));
            if (r0 < s.rows * group) return AttendSeg{s, b, first, last, end - begin};
        }
        return g;
    };
    // 64 pages of this wave, every fourth from i0 on: their numbers (-1: none)
    const auto page_ids = [&](const AttendSeg &g, int i0) {
        const int i = i0 + 4 * lane;
        int id = -1;
        if (i < g.last && i < (g.s.len + PAGE_POS - 1) / PAGE_POS) id = a.table[(size_t)g.s.slot * a.max_blocks + i];
        return (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
    };
    // A page's bytes are requested a page ahead: K's as soon as a page's scores are out, V's as its products go by, the first page's of the next
    // sequence before the waves' sums of this one meet.  (A page that is none: page 0's bytes, and none of its positions is seen.)
    KBytes kc[4];
    u32x4 vc[FB], vs[FB];
    uint32_t ks;
    const auto block_of = [&](int page) { return (size_t)(page < 0 ? 0 : page) * a.c.heads + head; };
    const auto take_k = [&](size_t block) {
#pragma unroll
        for (int t = 0; t < 4; ++t) kc[t] = *(const KBytes *)((a.c.k + block * (PAGE_POS * DH / 2) + t * (DH / 2)) + k_off);
        ks = *(const uint32_t *)((a.c.k_scale + block * (FB * PAGE_POS)) + ks_off);
    };
    const auto take_v = [&](size_t block, int j) {
        vc[j] = *(const u32x4 *)((a.c.v + block * (PAGE_POS * DH / 2) + 16 * j * PAGE_POS) + v_off);
        vs[j] = *(const u32x4 *)((a.c.v_scale + (block * FB + j) * PAGE_POS) + 16 * kb);
    };
    const auto take_page = [&](int page) {
        take_k(block_of(page));
#pragma unroll
        for (int j = 0; j < FB; ++j) take_v(block_of(page), j);
    };

    AttendSeg seg = segment(uniform(count_le(starts, n_seqs + 1, p0) - 1));
    AttendQ<DH, NT> qr;
    int id = -1;
    if (seg.last > 0) {
        id = page_ids(seg, seg.first + wave);
        attend_load_q<DH, NT, TYPE, DH / 32>(a, seg.s, head, group, r0, qr);
        if (seg.first + wave < seg.last) take_page(__builtin_amdgcn_readlane(id, 0));
    }
    while (seg.last > 0) {
        const AttendSeq s = seg.s;
#pragma unroll
        for (int u = 0; u < (PIECES + 255) / 256; ++u)
#pragma unroll
            for (int h = 0; h < (TYPE == ROWS_F32 ? 2 : 1); ++h) qr.raw[u][h] ^= turn;
        __syncthreads();
        attend_put_q<DH, NT, NQ, TYPE>(qr, q);
        if constexpr (TYPE == ROWS_F16)
#pragma unroll
            for (int u = 0; u < (PIECES + 255) / 256; ++u)
                if (u * 256 + (int)threadIdx.x < PIECES) q[NQ * PIECES + u * 256 + threadIdx.x] = qr.raw[u][0];
        __syncthreads();
        const AttendSeg after = segment(seg.b + 1);
        int id_after = -1;
        if (after.last > 0) {
            id_after = page_ids(after, after.first + wave);
            attend_load_q<DH, NT, TYPE, DH / 32>(a, after.s, head, group, r0, qr);
        }
        // the last position that every column sees, and each lane's columns' own
        const int seen = s.seen;
        int limit[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = r0 + 16 * n + col;
            limit[n] = r < s.rows * group ? seen + r / group : -1;
        }
        f32x4 o[NT][DT];
        float m[NT], l[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = LLMA_NEG_INF;
            l[n] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[n][d] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        // (pages behind the tile's last row are not seen by any of it)
        const int r_last = (r0 + 16 * NT < s.rows * group ? r0 + 16 * NT : s.rows * group) - 1, furthest = seen + r_last / group;
        const int stop = furthest < 0 ? 0 : seg.last < furthest / PAGE_POS + 1 ? seg.last : furthest / PAGE_POS + 1;
        for (int i0 = seg.first + wave; i0 < stop; i0 += 256) {
            const int n_here = (stop - i0 + 3) / 4 < 64 ? (stop - i0 + 3) / 4 : 64;
            for (int it = 0; it < n_here; ++it) {
                const int page = __builtin_amdgcn_readlane(id, it), base = (i0 + 4 * it) * PAGE_POS;
                const size_t next = block_of(__builtin_amdgcn_readlane(id, it + 1 < n_here ? it + 1 : it));      // (the last page's once more: no branch around the loads)
                // (several tiles' queries come from LDS for every page: kept in registers across pages they would push the sums out)
                int ql = lane;
                if constexpr (NT > 1) asm volatile("" : "+v"(ql));
                f32x4 sc[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < 4; ++t) sc[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
                const float k_by[4] = {scale_byte<0>(ks), scale_byte<1>(ks), scale_byte<2>(ks), scale_byte<3>(ks)};
                // (fp16 rows: one product of fp16 where K's scales allow it, two of bf16 otherwise; both exact)
                if (TYPE == ROWS_F16 && __ballot(!half_scales(ks)) == 0) {
#pragma unroll
                    for (int st = 0; st < STEPS; ++st)
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const u32x4 w = widen8_half(kc[t][st], k_by[t]);
#pragma unroll
                            for (int n = 0; n < NT; ++n) sc[n][t] = mfma16x16x32_half(w, q[NQ * PIECES + (n * STEPS + st) * 64 + ql], sc[n][t]);
                        }
                } else
#pragma unroll
                for (int st = 0; st < STEPS; ++st)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const u32x4 w = widen8(kc[t][st], k_by[t]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int pl = NQ - 1; pl >= 0; --pl) sc[n][t] = mfma16x16x32(w, q[pl * PIECES + (n * STEPS + st) * 64 + ql], sc[n][t]);
                    }
                __builtin_amdgcn_sched_barrier(0);
                take_k(next);
                __builtin_amdgcn_sched_barrier(0);
                const bool masked = page < 0 || base + PAGE_POS - 1 > seen;
                u32x4 nans[FB];
                uint32_t any = 0;
                if (masked) {
                    asm volatile("");                            // (a branch, not 150 selections for every page)
                    const int there = page < 0 ? 0 : s.len - base - 16 * kb;       // of the lane's 16 positions of V
                    // what lies behind the last position may be anything, and a NaN that only later rows see must not reach the others through 0 * NaN
#pragma unroll
                    for (int j = 0; j < FB; ++j)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t c = vs[j][w] & bytes_below(there - 4 * w), x = nan_scales(c);
                            any |= x;
                            nans[j][w] = x;
                            vs[j][w] = c & ~(x | (x - (x >> 7)));
                        }
                }
                u32x4 pb[NT][NP][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float x[16], top = LLMA_NEG_INF;
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = sc[n][e % 4][e / 4];
                    if (masked) {
                        asm volatile("");                        // (a branch, not selections for every page)
                        const int left = (page < 0 ? -1 : limit[n]) - base - 16 * kb;
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = e > left ? LLMA_NEG_INF : x[e];
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, x[e]);
                    top = fmaxf(top, lane_xor<16>(top));
                    top = fmaxf(top, lane_xor<32>(top)) * by;
                    // the reference of the exponentials moves only when a maximum passes it by 2^8: once or twice a sequence instead of the sums' 32 products a page
                    if (__ballot(top > m[n] + 8.f) != 0) {
                        const float mn = fmaxf(m[n], top), keep = __builtin_amdgcn_exp2f(m[n] - (mn == LLMA_NEG_INF ? 0.f : mn));
                        m[n] = mn;
                        l[n] *= keep;
#pragma unroll
                        for (int d = 0; d < DT; ++d) o[n][d] *= keep;
                    }
                    const float ref = m[n] == LLMA_NEG_INF ? 0.f : m[n];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], by, -ref));
                        l[n] += x[e];
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            float y = x[8 * u + 2 * w], z = x[8 * u + 2 * w + 1];
#pragma unroll
                            for (int pl = 0; pl < NP; ++pl) {
                                pb[n][pl][u][w] = bf16_pair(y, z);
                                if (pl + 1 < NP) { y -= __uint_as_float(pb[n][pl][u][w] << 16); z -= __uint_as_float(pb[n][pl][u][w] & 0xffff0000u); }
                            }
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (masked && __ballot(any != 0) != 0) attend_mx_nans<DH, NT>(nans, base, limit, o);
#pragma unroll
                for (int j = 0; j < FB; ++j) {
                    u32x4 even[2], odd[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) widen_v(vc[j], vs[j], u, even[u], odd[u]);
                    take_v(next, j);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                o[n][2 * j] = mfma16x16x32(even[u], pb[n][pl][u], o[n][2 * j]);
                                o[n][2 * j + 1] = mfma16x16x32(odd[u], pb[n][pl][u], o[n][2 * j + 1]);
                            }
                }
            }
            if (i0 + 256 < stop) {                               // (a share of more than 256 pages of one sequence)
                id = page_ids(seg, i0 + 256);
                take_page(__builtin_amdgcn_readlane(id, 0));
            }
        }
        id = id_after;
        if (after.last > 0 && after.first + wave < after.last) take_page(__builtin_amdgcn_readlane(id, 0));
        // ---- the waves' sums meet
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] += lane_xor<16>(l[n]);
            l[n] += lane_xor<32>(l[n]);
            if (kb == 0) { ml[wave][0][n * 16 + col] = m[n]; ml[wave][1][n * 16 + col] = l[n]; }
        }
        __syncthreads();
        float top[NT], sum[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float *const am = &ml[0][0][n * 16 + col];
            top[n] = fmaxf(fmaxf(am[0], am[2 * NT * 16]), fmaxf(am[4 * NT * 16], am[6 * NT * 16]));
            const float ref = top[n] == LLMA_NEG_INF ? 0.f : top[n];
            sum[n] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) sum[n] += am[(2 * w + 1) * NT * 16] * __builtin_amdgcn_exp2f(am[2 * w * NT * 16] - ref);
            const float f = __builtin_amdgcn_exp2f(m[n] - ref);
#pragma unroll
            for (int d = 0; d < DT; ++d) osum[((wave * NT + n) * DT + d) * 64 + lane] = o[n][d] * f;
        }
        __syncthreads();
        const bool whole = seg.first == 0 && seg.last == seg.pages;
        // the part's place: a share has at most one sequence that began before it (0) and one that goes on behind it (1)
        const int64_t at = (((int64_t)share * 2 + (seg.first == 0)) * a.c.heads + head) * plan.tiles + tile;
        float *const po = (float *)a.work + (a.n_seqs + 1 + 63) / 64 * 64;
        float *const pm = po + attend_parts(plan, a.c.heads) * 16 * NT * DH, *const pl = pm + attend_parts(plan, a.c.heads) * 16 * NT;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = r0 + 16 * n + col;
            if (r >= s.rows * group) continue;
            const int row = s.row0 + r / group, h = head * group + r % group;
            const float inv = sum[n] == 0.f ? 0.f : 1.f / sum[n];
#pragma unroll
            for (int u = 0; u < DT / 4; ++u) {
                // block jj's features 8 kb + 4 hf .. + 3: two of the even operand's, two of the odd one's
                const int jj = (4 * u + wave) / 2, hf = wave % 2, d = 32 * jj + 8 * kb + 4 * hf;
                typedef __attribute__((ext_vector_type(2))) float f32x2_t;
                f32x2_t e = (f32x2_t){0.f, 0.f}, f = e;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x2_t *const from_w = (const f32x2_t *)&osum[((w * NT + n) * DT + 2 * jj) * 64 + lane] + hf;
                    e += from_w[0];
                    f += from_w[2 * 64];
                }
                const f32x4 v = (f32x4){e[0], f[0], e[1], f[1]};
                if (whole) attend_store<TYPE>(a, row, h, d, v * inv);
                else *(f32x4 *)(po + (at * 16 * NT + 16 * n + col) * DH + d) = v;
            }
            if (!whole && wave == 0 && kb == 0) { pm[at * 16 * NT + 16 * n + col] = top[n]; pl[at * 16 * NT + 16 * n + col] = sum[n]; }
        }
        seg = after;
    }
}

// ---- many rows -----------------------------------------------------------------------------------
// fp16 products keep the sums of each block of 32 features in units of a power of two, `now` its exponent plus 127, so that V fits: a code of 0.5 .. 6 times 2^-23 ..
// 2^12 is exact in fp16.
// A page whose largest scale of the block lies outside 2^-8 .. 2^12 units makes that the unit, but none more than 2^60 below the largest before it (up to 2^62 units
// may have been added up, and fp32 ends at 2^128); and where a scale of the block lies below 2^-23 units, the unit goes down until the largest is 2^12.  So V loses
// bits where its scale is more than 2^35 below the largest of the block in its page, or more than 2^75 below 1 or another page's (the last bit 2^5 further down).
struct BlockUnit { int now, least; };
__device__ __forceinline__ void unit_for(int most, int fewest, BlockUnit &u) {   // the largest scale, 0 for none, and the smallest
    const bool other = ((unsigned)(most - u.now + 8) > 20u) & (most > 0);
    u.now = other ? most : u.now;
    const bool wide = (fewest - u.now < -23) & (most > 0);
    u.now = wide ? most - 12 : u.now;
    u.now = u.now > u.least ? u.now : u.least;
    u.least = u.now - 60 > u.least ? u.now - 60 : u.least;
}
// as widen_v, in fp16 and in units: by[t] for the word's four positions
__device__ __forceinline__ void widen_word_half(uint32_t w, const float *by, uint32_t (&even)[2], uint32_t (&odd)[2]) {
    const uint32_t p0 = widen2_half<0>(w, by[0]), p1 = widen2_half<1>(w, by[1]), p2 = widen2_half<2>(w, by[2]), p3 = widen2_half<3>(w, by[3]);
    even[0] = __builtin_amdgcn_perm(p1, p0, 0x05040100u);
    odd[0] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
    even[1] = __builtin_amdgcn_perm(p3, p2, 0x05040100u);
    odd[1] = __builtin_amdgcn_perm(p3, p2, 0x07060302u);
}
// The blocks of 64 NT rows of all sequences, each with the pages that it sees, lie end to end as a list of pages, per key head; equal shares of the list go to two workgroups per
// compute unit.  A block that lies in one share is finished there, the others' parts are joined by attend_mx_rows_join_kernel.  (Where there are many blocks a workgroup takes one,
// the longest first.)
struct RowsPlan { int blocks, shares; };                         // blocks: of the call's longest sequence; shares per key head, 0: a workgroup per block
#define ROWS_LISTED 2048         // blocks of a list, of which every workgroup makes the sums
#define ROWS_MIN_PAGES 4         // of a share
static RowsPlan rows_plan(int n_seqs, int max_blocks, int n_heads, int kv_heads, int max_rows, int rows) {
    RowsPlan p;
    p.blocks = (int)(((int64_t)max_rows * (n_heads / kv_heads) + rows - 1) / rows);
    const int64_t listed = (int64_t)p.blocks * n_seqs, pages = listed * max_blocks, most = (pages + ROWS_MIN_PAGES - 1) / ROWS_MIN_PAGES;
    int64_t shares = 2 * ATTEND_CUS / kv_heads;
    shares = shares < 1 ? 1 : shares;
    const bool small = max_blocks <= 8 && listed * kv_heads >= 128;      // (blocks enough, and so short that a share's several starts cost more than an uneven end)
    // (pages of the list, and those up to the last share's end, are counted in 32 bits)
    p.shares = listed > ROWS_LISTED || pages > 0x7fffffff - 2 * ATTEND_CUS || small ? 0 : (int)(shares < most ? shares : most);
    return p;
}
// work: [pages before every block of the list, rounded up to 64 ints][parts' O][parts' m][parts' l]
__host__ __device__ static inline int64_t rows_head(const RowsPlan &p, int n_seqs) { return ((int64_t)p.blocks * n_seqs + 1 + 63) / 64 * 64; }
__host__ __device__ static inline int64_t rows_parts(const RowsPlan &p, int kv_heads) { return (int64_t)p.shares * 2 * kv_heads; }
// Prompts: a workgroup takes 64 NT rows of a sequence's key head and pages that they see.  Each page is widened once, for all four waves, into LDS as the operands'
// images (16 KB of K, 16 KB of V at head_dim 128): wave t has score tile t, and block t of V's features (of two blocks at head_dim 64: half of one's positions).  A
// page is requested two ahead, widened one ahead, one barrier a page.  The rest is as with 8 bits: a wave holds its rows' queries and sums in registers, pages behind
// its rows are skipped, and the reference of the exponentials moves only when a maximum passes it by 2^8.
// Bound by issue: two sequences of up to 2047 rows, 32 query and 8 key heads of 128, over up to 2900 positions before, bf16, 136 GFLOP in 258 us and 17 for the join =
// 0.49 PFLOP/s.  A workgroup per block left the compute units empty for 30 % of the time (310 us); what is left is the products (a third of the cycles) and the vector
// instructions (half), which hardly overlap.  Wave priorities, by phase or by wave, changed nothing.
// bf16 rows' probabilities are one plane of fp16: with two of bf16, inside a captured graph, 284 us where both launches now take 247, and outputs 1.660e-3 (rms,
// relative to 64 bits) off, which is their own rounding, where they are 1.670e-3.
// (fp16 rows at head_dim 128: the second plane of queries costs 132 bytes of scratch a lane)
template <int DH> constexpr int rows_images = (4 * (DH / 32) + (DH / 16) * 2) * 64;          // 16-byte pieces of a page
template <int DH, int NT, int TYPE>
__global__ __launch_bounds__(256, 2) void attend_mx_rows_kernel(AttendMxArgs a, RowsPlan plan) {
    constexpr bool HALF = TYPE == ROWS_BF16;
    constexpr float BIAS = HALF ? 7.f : 0.f;
    constexpr int NQ = attend_nq<TYPE>, NP = attend_np<TYPE, HALF>, STEPS = DH / 32, FB = DH / 32, DT = DH / 16;
    constexpr int KI = 4 * STEPS, VI = DT * 2;                   // images of K, of V
    constexpr int US = FB / 2;                                   // operand pairs of V a wave widens (positions 8 u .. of a lane's 16)
    typedef std::conditional_t<DH == 128, u32x4, u32x2> KBytes;
    extern __shared__ u32x4 lds[];                               // [2] pages
    __shared__ int nan_seen[2][4];
    __shared__ uint32_t units[2];                                // a byte a wave: of the page's images
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ int part[4];
    int *const starts = (int *)(lds + 2 * rows_images<DH>);      // pages before every block of the list, and of all
    const int head = blockIdx.x % a.c.heads, rest = blockIdx.x / a.c.heads, group = a.n_heads / a.c.heads;
    const int listed = plan.shares > 0 ? plan.blocks * a.n_seqs : 1;
    // pages that a block sees; one for a block that sees nothing (its rows become 0), none for one that is not there
    const auto pages_of = [&](const AttendSeq &s, int r0) {
        const int R = s.rows * group, r1 = r0 + 64 * NT < R ? r0 + 64 * NT : R, furthest = s.seen + (r1 - 1) / group;
        return r0 >= R ? 0 : furthest < 0 ? 1 : furthest / PAGE_POS + 1;
    };
    int from = 0, to, g;                                         // pages of the list, the block that the first is in
    if (plan.shares > 0) {
        int total = 0;
        for (int g0 = 0; g0 < listed; g0 += 256) {
            const int i = g0 + threadIdx.x;
            int sum, pages = 0;
            if (i < listed) pages = pages_of(attend_seq(a, i / plan.blocks), i % plan.blocks * 64 * NT);
            const int at = block_scan<4>(pages, part, &sum);
            if (i < listed) starts[i] = total + at;
            total += sum;
        }
        if (threadIdx.x == 0) starts[listed] = total;
        __syncthreads();
        if (blockIdx.x == 0)                                     // (for attend_mx_rows_join_kernel)
            for (int i = threadIdx.x; i <= listed; i += 256) ((int *)a.work)[i] = starts[i];
        total = uniform(total);
        int per = (total + plan.shares - 1) / plan.shares;
        per = per < ROWS_MIN_PAGES ? ROWS_MIN_PAGES : per;
        if ((int64_t)rest * per >= total) return;
        from = rest * per;
        to = from + per < total ? from + per : total;
        g = uniform(count_le(starts, listed + 1, from) - 1);
    } else {
        g = (plan.blocks - 1 - rest / a.n_seqs) + rest % a.n_seqs * plan.blocks;
        to = pages_of(uniform(attend_seq(a, g / plan.blocks)), g % plan.blocks * 64 * NT);
    }
  for (; from < to; ++g) {
    const int b = g / plan.blocks, r0 = g % plan.blocks * 64 * NT;
    const AttendSeq s = uniform(attend_seq(a, b));
    const int R = s.rows * group, seen = s.seen;
    const int begin = plan.shares > 0 ? uniform(starts[g]) : 0, all_pages = plan.shares > 0 ? uniform(starts[g + 1]) - begin : to;
    const int p_first = from - begin, pages = to - begin < all_pages ? to - begin : all_pages;       // the block's pages here: p_first .. pages - 1
    if (p_first >= pages) continue;
    from = begin + pages;
    const int kb = lane >> 4, col = lane & 15, w0 = r0 + wave * 16 * NT;
    const int w1 = w0 + 16 * NT < R ? w0 + 16 * NT : R;
    const int wave_first = w0 < R ? seen + w0 / group : -1, wave_last = w0 < R ? seen + (w1 - 1) / group : -1, block_first = seen + r0 / group;
    const int vj = FB == 4 ? wave : wave / 2, u0 = FB == 4 ? 0 : wave % 2;       // the wave's block of V, its first operand pair
    const uint32_t k_off = (4 * col + wave) * (DH / 2) + kb * (DH / 8), ks_off = (kb * FB / 4) * PAGE_POS + 4 * col + wave;
    const uint32_t v_off = (16 * vj + col) * PAGE_POS + 16 * kb, vs_off = vj * PAGE_POS + 16 * kb;
    // ---- the wave's queries.  A negative scale turns their signs, so that the largest score is the largest product
    u32x4 q[NQ][NT][STEPS];
    const uint32_t turn = a.scale < 0.f ? 0x80008000u : 0u;
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = w0 + 16 * n + col;
        limit[n] = r < R ? seen + r / group : -1;
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            float v[8];
#pragma unroll
            for (int p = 0; p < NQ; ++p) q[p][n][t] = (u32x4){0, 0, 0, 0};
            if (r < R) {
                const int row = s.row0 + r / group, hq = head * group + r % group, d = (DH / 4) * kb + 8 * t;
                row8<TYPE>(a.q, (int64_t)row * a.q_row + hq * a.q_head + d, v);
#pragma unroll
                for (int p = 0; p < NQ; ++p)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t x = bf16_pair(v[2 * w], v[2 * w + 1]);
                        q[p][n][t][w] = x ^ turn;
                        v[2 * w] -= __uint_as_float(x << 16);
                        v[2 * w + 1] -= __uint_as_float(x & 0xffff0000u);
                    }
            }
        }
    }
    // ---- page numbers, 64 pages a lane at a time: the present 64 and the next
    const auto pages_from = [&](int i0) {
        const int i = i0 + lane;
        int id = -1;
        if (i < pages && i * PAGE_POS < s.len) id = a.table[(size_t)s.slot * a.max_blocks + i];      // (a sequence without positions may be one without a slot)
        return (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
    };
    int now = pages_from(p_first), later = pages_from(p_first + 64), now_at = p_first;           // now_at: the first page of `now`
    const auto id_of = [&](int i) { return i < now_at + 64 ? __builtin_amdgcn_readlane(now, i - now_at) : __builtin_amdgcn_readlane(later, i - now_at - 64); };
    // a thread's share of a page
    KBytes kc;
    u32x4 vc, vs;
    uint32_t ks;
    const auto take = [&](int i) {
        const int id = id_of(i);
        const size_t at = (size_t)(id < 0 ? 0 : id) * a.c.heads + head;
        kc = *(const KBytes *)(a.c.k + at * (PAGE_POS * DH / 2) + k_off);
        ks = *(a.c.k_scale + at * (FB * PAGE_POS) + ks_off);
        vc = *(const u32x4 *)(a.c.v + at * (PAGE_POS * DH / 2) + v_off);
        vs = *(const u32x4 *)(a.c.v_scale + at * (FB * PAGE_POS) + vs_off);
    };
    BlockUnit unit{127, 67};                                     // of the wave's block, of the page that was widened last
    const auto widen = [&](int i) {
        u32x4 *const to = lds + (i & 1) * rows_images<DH> + lane;
        const float k_by = __uint_as_float(ks << 23);
#pragma unroll
        for (int t = 0; t < STEPS; ++t) to[(wave * STEPS + t) * 64] = widen8(kc[t], k_by);
        const bool masked = i * PAGE_POS + PAGE_POS - 1 > block_first || id_of(i) < 0;           // positions that some row does not see
        uint32_t any = 0;
        if (masked) {
            asm volatile("");
            const int there = id_of(i) < 0 ? 0 : s.len - i * PAGE_POS - 16 * kb;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t is = vs[w] & bytes_below(there - 4 * w), nan = nan_scales(is);
                any |= nan;
                vs[w] = is & ~(nan | (nan - (nan >> 7)));
            }
        }
        any = __ballot(any != 0) != 0;
        if (lane == 0) nan_seen[i & 1][wave] = (int)any;
        bool plain = true;                                       // units of 1, and no scale that is not one of them: the scales as they lie
        if constexpr (HALF) {
            // (lanes of a group have the same 16 scales: each looks at four.  Bytes above 139, from 1 to 103; bytes of 119 and more)
            const uint32_t x = col & 2 ? (col & 1 ? vs[3] : vs[2]) : (col & 1 ? vs[1] : vs[0]), low = x & 0x7f7f7f7fu;
            const uint32_t above = (low + 0x74747474u) & x, below = ((low + 0x7f7f7f7fu) | x) & ~((low + 0x18181818u) | x);
            plain = unit.now == 127 && __ballot(((above | below) & 0x80808080u) != 0) == 0 && __ballot((((low + 0x09090909u) | x) & 0x80808080u) != 0) != 0;
        }
        float half_by[4 * 2 * US];                               // of fp16's positions
        if constexpr (HALF) {
            const auto byte_of = [&](int t) { const uint32_t x = FB == 4 ? vs[t / 4] : u0 ? vs[2 + t / 4] : vs[t / 4]; return x >> 8 * (t % 4) & 255u; };
            if (plain) {
#pragma unroll
                for (int h = 0; h < 2 * US; ++h) {
                    const uint32_t x = FB == 4 ? vs[h] : u0 ? vs[2 + h] : vs[h];
                    half_by[4 * h] = scale_byte<0>(x);
                    half_by[4 * h + 1] = scale_byte<1>(x);
                    half_by[4 * h + 2] = scale_byte<2>(x);
                    half_by[4 * h + 3] = scale_byte<3>(x);
                }
            } else {
                uint32_t most = 0, fewest = 254;                 // (0: a position that is not there, or 2^-127)
#pragma unroll
                for (int w = 0; w < 4; ++w)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint32_t e = vs[w] >> 8 * t & 255u;
                        most = e > most && e != 255u ? e : most;
                        fewest = e < fewest && e != 0u ? e : fewest;
                    }
                most = max((int)most, lane_xor<16>((int)most));
                most = max((int)most, lane_xor<32>((int)most));
                fewest = min((int)fewest, lane_xor<16>((int)fewest));
                fewest = min((int)fewest, lane_xor<32>((int)fewest));
                unit_for(uniform((int)most), uniform((int)fewest), unit);
#pragma unroll
                for (int t = 0; t < 8 * US; ++t) {
                    const int raw = (int)byte_of(t), e = raw - unit.now + 127;
                    half_by[t] = __uint_as_float((uint32_t)(raw == 255 ? 255 : e > 0 ? e : 0) << 23);
                }
            }
            if (lane == 0) ((uint8_t *)&units[i & 1])[wave] = (uint8_t)unit.now;
        }
#pragma unroll
        for (int k = 0; k < US; ++k) {
            const int u = u0 + k;
            u32x4 even, odd;
            if constexpr (HALF) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t c = FB == 4 ? vc[2 * k + h] : u0 ? vc[2 + h] : vc[h];
                    uint32_t e2[2], o2[2];
                    widen_word_half(c, half_by + 4 * (2 * k + h), e2, o2);
                    even[2 * h] = e2[0];
                    even[2 * h + 1] = e2[1];
                    odd[2 * h] = o2[0];
                    odd[2 * h + 1] = o2[1];
                }
            } else if constexpr (FB == 4) widen_v(vc, vs, k, even, odd);
            else {
                const u32x4 c = u0 ? (u32x4){vc[2], vc[3], 0, 0} : (u32x4){vc[0], vc[1], 0, 0}, x = u0 ? (u32x4){vs[2], vs[3], 0, 0} : (u32x4){vs[0], vs[1], 0, 0};
                widen_v(c, x, 0, even, odd);
            }
            to[(KI + 2 * (2 * vj) + u) * 64] = even;
            to[(KI + 2 * (2 * vj + 1) + u) * 64] = odd;
        }
    };
    f32x4 o[NT][DT];
    float m[NT];
    f32x4 l[NT];                                                 // the rows' sums, by products with ones
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = LLMA_NEG_INF;
        l[n] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    // (not 0: minus infinity has to stay that)
    const float by = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 1e-37f);
    take(p_first);
    widen(p_first);
    if (p_first + 1 < pages) take(p_first + 1);
    __syncthreads();
    uint32_t o_units = 0x7f7f7f7fu;                              // that the wave's sums are in
    for (int i = p_first; i < pages; ++i) {
        if (i + 1 < pages) widen(i + 1);
        if (i + 2 < pages) take(i + 2);
        const int base = i * PAGE_POS;
        if (base <= wave_last) {                                 // (the wave's rows see some of it)
            // operands come from LDS eight ahead of their products, V's first ones behind K's last
            const u32x4 *const img = lds + (i & 1) * rows_images<DH> + lane;
            u32x4 w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = img[j * 64];
            const int id = id_of(i);
            const bool masked = id < 0 || base + PAGE_POS - 1 > wave_first;
            u32x4 pb[NT][NP][2];
            f32x4 sc[NT][4];
            if constexpr (HALF) {
                const uint32_t page_units = uniform((int)units[i & 1]);
                if (page_units != o_units) {                     // (exact)
#pragma unroll
                    for (int j = 0; j < FB; ++j) {
                        const int to = (int)(o_units >> 32 / FB * j & 255u) - (int)(page_units >> 32 / FB * j & 255u);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            o[n][2 * j] = times_pow2(o[n][2 * j], to);
                            o[n][2 * j + 1] = times_pow2(o[n][2 * j + 1], to);
                        }
                    }
                    o_units = page_units;
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < 4; ++t) sc[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int j = 0; j < KI; ++j) {
                const int t = j / STEPS, st = j % STEPS;
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p)
#pragma unroll
                    for (int n = 0; n < NT; ++n) sc[n][t] = mfma16x16x32(w[j % 8], q[p][n][st], sc[n][t]);
                w[j % 8] = img[(j + 8) * 64];
                __builtin_amdgcn_sched_group_barrier(0x008, NT * NQ, 0);       // (products, then a load: as written)
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_s_setprio(0);
            // position e of the lane's 16: tile e % 4, register e / 4
            if (masked) {
                asm volatile("");                                // (a branch: as selections this would cost every page 32 comparisons a tile)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int left = (id < 0 ? -1 : limit[n]) - base - 16 * kb;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[n][e % 4][e / 4] = e > left ? LLMA_NEG_INF : sc[n][e % 4][e / 4];
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float top = LLMA_NEG_INF;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[n][t][r]);
                top = fmaxf(top, lane_xor<16>(top));
                top = fmaxf(top, lane_xor<32>(top)) * by;
                if (__ballot(top > m[n] + (8.f + BIAS)) != 0) {
                    const float mn = fmaxf(m[n], top - BIAS), keep = __builtin_amdgcn_exp2f(m[n] - (mn == LLMA_NEG_INF ? 0.f : mn));
                    m[n] = mn;
                    l[n] *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] *= keep;
                }
                const float ref = m[n] == LLMA_NEG_INF ? 0.f : m[n];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int r = 2 * u + w / 2, t = 2 * (w & 1);
                        float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][t][r], by, -ref)), z = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][t + 1][r], by, -ref));
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            pb[n][p][u][w] = HALF ? half_pair(y, z) : bf16_pair(y, z);
                            if (p + 1 < NP) { y -= __uint_as_float(pb[n][p][u][w] << 16); z -= __uint_as_float(pb[n][p][u][w] & 0xffff0000u); }
                        }
                    }
            }
            // (taken out of the image where the block's first row does not see all of the page: also for waves whose rows all do)
            if (base + PAGE_POS - 1 > block_first && (nan_seen[i & 1][0] | nan_seen[i & 1][1] | nan_seen[i & 1][2] | nan_seen[i & 1][3])) {
                u32x4 nans[FB];
                const size_t at = (size_t)(id < 0 ? 0 : id) * a.c.heads + head;
                const int there = id < 0 ? 0 : s.len - base - 16 * kb;
#pragma unroll
                for (int j = 0; j < FB; ++j) {
                    nans[j] = *(const u32x4 *)(a.c.v_scale + (at * FB + j) * PAGE_POS + 16 * kb);
#pragma unroll
                    for (int w = 0; w < 4; ++w) nans[j][w] = nan_scales(nans[j][w] & bytes_below(there - 4 * w));
                }
                attend_mx_nans<DH, NT>(nans, base, limit, o);
            }
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        l[n] = HALF ? mfma16x16x32_half((u32x4){0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u}, pb[n][p][u], l[n])
                                    : mfma16x16x32((u32x4){0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}, pb[n][p][u], l[n]);
#pragma unroll
            for (int j = 0; j < VI; ++j) {
                const int d = j / 2, u = j % 2;
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][d] = HALF ? mfma16x16x32_half(w[(KI + j) % 8], pb[n][p][u], o[n][d]) : mfma16x16x32(w[(KI + j) % 8], pb[n][p][u], o[n][d]);
                if (j + 8 < VI) {
                    w[(KI + j) % 8] = img[(KI + j + 8) * 64];
                    __builtin_amdgcn_sched_group_barrier(0x008, NT * NP, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if (i + 1 == now_at + 64) {
            now = later;
            now_at += 64;
            later = pages_from(now_at + 64);
        }
        __syncthreads();
    }
    const bool whole = p_first == 0 && pages == all_pages;
    // the part's place: a share has at most one block that began before it (0) and one that goes on behind it (1)
    const int64_t at = (((int64_t)rest * 2 + (p_first == 0)) * a.c.heads + head) * (64 * NT) + wave * 16 * NT;
    float *const po = (float *)a.work + rows_head(plan, a.n_seqs), *const pm = po + rows_parts(plan, a.c.heads) * 64 * NT * DH, *const pl = pm + rows_parts(plan, a.c.heads) * 64 * NT;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = w0 + 16 * n + col;
        if (r >= R) continue;
        const float inv = !whole ? 1.f : l[n][0] == 0.f ? 0.f : 1.f / l[n][0];
        if (!whole && kb == 0) {
            pm[at + 16 * n + col] = m[n];
            pl[at + 16 * n + col] = l[n][0];
        }
#pragma unroll
        for (int j = 0; j < FB; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 v = (f32x4){o[n][2 * j][2 * h], o[n][2 * j + 1][2 * h], o[n][2 * j][2 * h + 1], o[n][2 * j + 1][2 * h + 1]} * inv;
                if constexpr (HALF) v = times_pow2(v, (int)(o_units >> 32 / FB * j & 255u) - 127);
                const int d = 32 * j + 8 * kb + 4 * h;
                if (whole) attend_store<TYPE>(a, s.row0 + r / group, head * group + r % group, d, v);
                else *(f32x4 *)(po + (at + 16 * n + col) * DH + d) = v;
            }
    }
  }
}
// rows of blocks that lie in several shares, JOIN_ROWS a workgroup; a thread has four features of several rows, whose parts are requested together, or of one row whose
// many parts are
template <int DH, int TYPE, int JOIN_ROWS>
__global__ __launch_bounds__(256) void attend_mx_rows_join_kernel(AttendMxArgs a, RowsPlan plan, int rows) {
    constexpr int LANES = DH / 4, EACH = JOIN_ROWS * LANES / 256, AHEAD = EACH == 1 ? 8 : 2;
    const int group = a.n_heads / a.c.heads, b = blockIdx.z, head = blockIdx.y, r0 = blockIdx.x * JOIN_ROWS, block = r0 / rows;
    const int *const starts = (const int *)a.work;
    const int g = b * plan.blocks + block, total = starts[plan.blocks * a.n_seqs], p0 = starts[g], p1 = starts[g + 1];
    int per = (total + plan.shares - 1) / plan.shares;
    per = per < ROWS_MIN_PAGES ? ROWS_MIN_PAGES : per;
    const int s0 = p0 / per, s1 = (p1 - 1) / per;
    if (p0 >= p1 || s0 == s1) return;
    const AttendSeq s = attend_seq(a, b);
    const float *const po = (const float *)a.work + rows_head(plan, a.n_seqs), *const pm = po + rows_parts(plan, a.c.heads) * rows * DH, *const pl = pm + rows_parts(plan, a.c.heads) * rows;
    const auto place = [&](int sh) { return (((int64_t)sh * 2 + (sh == s0)) * a.c.heads + head) * rows + r0 % rows; };
    const int d = threadIdx.x % LANES * 4, at = threadIdx.x / LANES;
    float m[EACH], l[EACH];
    f32x4 o[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        m[k] = LLMA_NEG_INF;
        l[k] = 0.f;
        o[k] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    // (rows behind the sequence's last have a place too: what lies there is read and not used)
#pragma unroll AHEAD
    for (int sh = s0; sh <= s1; ++sh)
#pragma unroll
        for (int k = 0; k < EACH; ++k) m[k] = fmaxf(m[k], pm[place(sh) + at + k * (JOIN_ROWS / EACH)]);
#pragma unroll AHEAD
    for (int sh = s0; sh <= s1; ++sh)
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int64_t i = place(sh) + at + k * (JOIN_ROWS / EACH);
            const float f = __builtin_amdgcn_exp2f(pm[i] - (m[k] == LLMA_NEG_INF ? 0.f : m[k]));
            l[k] += pl[i] * f;
            o[k] += *(const f32x4 *)(po + i * DH + d) * f;
        }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = r0 + at + k * (JOIN_ROWS / EACH);
        if (r < s.rows * group) attend_store<TYPE>(a, s.row0 + r / group, head * group + r % group, d, o[k] * (l[k] == 0.f ? 0.f : 1.f / l[k]));
    }
}

template <int DH, int NT, int TYPE>
static void launch_attend_nt(const AttendMxArgs &a, const AttendPlan &p, hipStream_t st) {
    const size_t bytes = (size_t)attend_mx_lds<DH, NT, TYPE> + (size_t)(a.n_seqs + 1) * 4;
    hipLaunchKernelGGL((attend_paged_mx_kernel<DH, NT, TYPE>), dim3((p.whole ? a.n_seqs : p.shares) * a.c.heads * p.tiles), dim3(256), bytes, st, a, p);
}
static AttendPlan attend_mx_plan(int n_seqs, int max_blocks, int n_heads, int kv_heads, int max_rows) {
    // Which sequences stay whole: the 8-bit cache's rule, with a page at what 70 bytes a position would cost, for each tile of rows, whatever its head_dim, and tables
    // of up to 64 pages.
    // us inside a captured graph, cut and whole (32 heads of 128, 9 rows; 8 of 64; 32 / 8 of 128, 5 rows):
    //          1 x 500    1 x 1001   1 x 1500   6 x 1001   6 x 3000   16 x 1001  64 x 1900 | 1 x 1001, 1 row  6 x 1300, 9  1 x 2000, 1  6 x 2400, 9 | 4 x 1001
    //   bf16   11.9 9.5   12.3 11.7  12.8 13.8  20.2 12.8  28.3 22.8  20.7 18.3  117 110   | 10.7 9.7         13.8 11.3    11.0 12.7    15.7 14.5   | 14.3 15.6
    //   fp32   12.5 10.5  12.8 13.7  13.6 17.0  21.9 14.9  32.1 28.9  24.3 21.7  129 128   | 11.0 10.9        14.7 13.2    11.4 15.0    16.7 17.6   | 16.4 19.7
    const int64_t r = (int64_t)max_rows * (n_heads / kv_heads);
    return attend_plan(n_seqs, max_blocks, n_heads, kv_heads, 70 * (r <= 16 ? 1 : r <= 32 ? 2 : r <= 48 ? 3 : 4), max_rows, 64);
}
template <int DH, int NT, int TYPE>
static void launch_attend_rows(const AttendMxArgs &a, hipStream_t st) {
    const RowsPlan p = rows_plan(a.n_seqs, a.max_blocks, a.n_heads, a.c.heads, a.max_rows, 64 * NT);
    const unsigned grid = p.shares > 0 ? (unsigned)p.shares * a.c.heads : (unsigned)p.blocks * a.n_seqs * a.c.heads;
    const size_t bytes = 2 * rows_images<DH> * 16 + (p.shares > 0 ? ((size_t)p.blocks * a.n_seqs + 1) * 4 : 0);
    hipLaunchKernelGGL((attend_mx_rows_kernel<DH, NT, TYPE>), dim3(grid), dim3(256), bytes, st, a, p);
    constexpr int ONE = 1024 / DH;                               // rows whose features fill a workgroup once
    if (p.shares > 4 * p.blocks * a.n_seqs) hipLaunchKernelGGL((attend_mx_rows_join_kernel<DH, TYPE, ONE>), dim3((unsigned)p.blocks * (64 * NT / ONE), a.c.heads, a.n_seqs), dim3(256), 0, st, a, p, 64 * NT);
    else if (p.shares > 1) hipLaunchKernelGGL((attend_mx_rows_join_kernel<DH, TYPE, 4 * ONE>), dim3((unsigned)p.blocks * (64 * NT / (4 * ONE)), a.c.heads, a.n_seqs), dim3(256), 0, st, a, p, 64 * NT);
}
template <int TYPE> constexpr int rows_nt = TYPE == ROWS_F32 ? 1 : 2;             // (three planes of queries and probabilities leave room for one tile)
// Which calls take the many-rows form: those with more rows a key head than the shares' kernel holds (64); at head_dim 64, whose pages are half as much work for the
// same start and end, from 6144 rows in all blocks on.  us inside a captured graph, here and in shares of the steps' kernel (sequences x positions before, rows, query
// / key heads):
//             head_dim 128                                                                                     head_dim 64
//         1 x 1000, 70, 8/8   1 x 8000, 20, 32/8   1 x 20000, 130, 8/8   64 x 1000, 20, 32/8   4 x 200, 100, 32/32   8 x 2000, 40, 16/2   30 x 60, 70, 8/8   1 x 4000, 500, 8/8   1 x 20000, 70, 8/8
//   bf16  21.9 26.7           31.0 35.4            47.8 57.8             54.5 130.3            18.7 28.3             25.8 29.0            12.6 18.9          36.3 27.3            44.0 25.6
//   fp16  25.2 27.5           34.5 37.2            56.7 61.8             73.0 140.3            24.3 29.6             27.5 30.5            13.1 19.9          38.5 29.0            46.5 27.3
//   fp32  23.2 29.9           33.5 43.3            60.8 73.6             87.0 167.3            17.3 36.0             31.1 34.0            11.9 21.9          36.4 32.8            37.0 31.3
// 49 .. 64 rows a key head stay with the steps' form, where bf16 rows' probabilities keep 16 bits and V its range.  Its fourth tile spills at head_dim 128 (296 / 460 /
// 316 bytes a lane in bf16 / fp16 / fp32; two tiles 28 in fp16, 64 in fp32), and but for single long sequences this form would be the faster one (head_dim 128, lengths
// up to what is named, here and there):
//         1 x 20000, 8/8   1 x 4000, 32/8   16 x 4096, 32/32   61 x 1500, 32/8   4 x 300, 32/32
//   48 rows  bf16  45.9 29.1        22.1 19.0        124 90             70.5 50.3         19.4 15.0
//            fp16  52.2 30.1        25.4 19.6        165 96             89.5 54.3         25.2 16.1
//            fp32  46.6 33.6        21.1 20.9        122 116            65.7 65.9         17.5 18.0
//   56 rows  bf16  45.9 43.8        22.5 27.8        126 151            71.4 84.1         19.5 26.0
//            fp16  53.3 51.4        26.0 31.8        167 192            91.0 107          25.3 30.6
//            fp32  47.9 52.7        22.0 31.7        127 197            67.3 107          17.8 29.8
#define ROWS_BLOCKS (1 << 23)    // of a launch: fewer
static int64_t rows_blocks(int n_seqs, int n_heads, int kv_heads, int max_rows, int rows) { return ((int64_t)max_rows * (n_heads / kv_heads) + rows - 1) / rows * n_seqs * kv_heads; }
static bool takes_rows(int n_seqs, int n_heads, int kv_heads, int dh, int max_rows, int rows) {
    const int64_t blocks = rows_blocks(n_seqs, n_heads, kv_heads, max_rows, rows);
    return (int64_t)max_rows * (n_heads / kv_heads) > 64 && (dh == 128 || blocks * rows >= 6144) && blocks < ROWS_BLOCKS;
}
template <int DH, int TYPE>
static void launch_attend_type(const AttendMxArgs &a, hipStream_t st) {
    if (takes_rows(a.n_seqs, a.n_heads, a.c.heads, DH, a.max_rows, 64 * rows_nt<TYPE>)) return launch_attend_rows<DH, rows_nt<TYPE>, TYPE>(a, st);
    const AttendPlan p = attend_mx_plan(a.n_seqs, a.max_blocks, a.n_heads, a.c.heads, a.max_rows);
    if (p.nt == 1) launch_attend_nt<DH, 1, TYPE>(a, p, st);
    else if (p.nt == 2) launch_attend_nt<DH, 2, TYPE>(a, p, st);
    else if (p.nt == 3) launch_attend_nt<DH, 3, TYPE>(a, p, st);
    else launch_attend_nt<DH, 4, TYPE>(a, p, st);
    if (p.shares > 1 && !p.whole)
        hipLaunchKernelGGL((attend_join_kernel<DH, TYPE, AttendMxArgs>), dim3((a.max_rows * (a.n_heads / a.c.heads) + 3) / 4, a.c.heads, a.n_seqs), dim3(256), 0, st, a, p);
}
int64_t attend_paged_mx_bytes(int n_seqs, int max_blocks, int n_heads, int kv_heads, int dh, int max_rows) {
    int64_t most = attend_bytes(attend_mx_plan(n_seqs, max_blocks, n_heads, kv_heads, max_rows), n_seqs, kv_heads, dh);
    for (int rows = 64; rows <= 128; rows += 64) {               // (fp32's row blocks, the others')
        // (a workspace for some number of sequences does for fewer: for the most that take this form, where more do not, and as if cut, where more are not)
        const int64_t many = (ROWS_BLOCKS - 1) / rows_blocks(1, n_heads, kv_heads, max_rows, rows);
        const int taken = many < n_seqs ? (int)many : n_seqs;
        if (!takes_rows(taken, n_heads, kv_heads, dh, max_rows, rows)) continue;
        RowsPlan p = rows_plan(1, max_blocks, n_heads, kv_heads, max_rows, rows);
        if (p.blocks > ROWS_LISTED) continue;
        const int listed = taken < ROWS_LISTED / p.blocks ? taken : ROWS_LISTED / p.blocks;
        p.shares = 2 * ATTEND_CUS / kv_heads > 0 ? 2 * ATTEND_CUS / kv_heads : 1;
        const int64_t bytes = (rows_head(p, listed) + (p.shares > 1 ? rows_parts(p, kv_heads) * rows * (dh + 2) : 0)) * 4;       // (one share a key head cuts nothing)
        most = bytes > most ? bytes : most;
    }
    return most;
}
void launch_attend_paged_mx(const AttendMxArgs &a, hipStream_t st) {
    if (a.n_seqs < 1 || a.n_rows < 1 || a.max_rows < 1) return;
    auto of = [&](auto dh) {
        constexpr int DH = decltype(dh)::value;
        if (a.type == ROWS_BF16) launch_attend_type<DH, ROWS_BF16>(a, st);
        else if (a.type == ROWS_F16) launch_attend_type<DH, ROWS_F16>(a, st);
        else launch_attend_type<DH, ROWS_F32>(a, st);
    };
    if (a.c.dh == 128) of(std::integral_constant<int, 128>{});
    else of(std::integral_constant<int, 64>{});
}
