// The paged 8-bit cache: pages and slots of a step, the write into the cache, attention of a step's rows over it.
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
// pages and slots of a step
// ---------------------------------------------------------------------------------------------
// need_b = ceil((len_b + rows_b) / 64) pages.  What a sequence owns beyond that goes back on the stack of free pages, in the reverse
// order of granting (a grant taken back leaves the stack as it was); what it lacks comes off the stack's top, sequence by sequence.
// Places are prefix sums, so the result does not depend on the order of execution.  One workgroup, a thread per sequence
// and then a thread per page and per row: all of it is a chain of dependent reads, a few microseconds however little there is to do.
// 16 sequences of 9 rows 3.9 us, 512 prompts of 130 rows (33 thousand) 5.6 and 5.0 for the rows in a launch of their own, of which an empty launch is 2.
#define MAP_THREADS 1024
#define MAP_ROWS_HERE 8192       // rows whose slots the same workgroup writes; more take a launch of many
#define MAP_MAX_SLOTS 65536      // (bits of LDS that find a slot listed twice)

// what is known of a sequence: of the workgroup's present 1024, and where they begin in three sums
struct MapSeq { int slot, len, rows, own, need; };
template <int N> struct MapTile { MapSeq seq[N]; int first[N]; };
struct MapSums { int back, more, rows; };

// exclusive prefix sums of three numbers over the workgroup's NW waves, *total the sums
template <int NW>
__device__ __forceinline__ MapSums block_scan3(MapSums v, MapSums *part, MapSums *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const MapSums in = {wave_scan(v.back), wave_scan(v.more), wave_scan(v.rows)};
    __syncthreads();
    if (lane == 63) part[wave] = in;
    __syncthreads();
    MapSums before{0, 0, 0}, all{0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const MapSums p = part[w];
        const int in_front = w < wave ? -1 : 0;
        before.back += p.back & in_front; before.more += p.more & in_front; before.rows += p.rows & in_front;
        all.back += p.back; all.more += p.more; all.rows += p.rows;
    }
    *total = all;
    return MapSums{before.back + in.back - v.back, before.more + in.more - v.more, before.rows + in.rows - v.rows};
}
// row i of the call, row j of sequence b
__device__ __forceinline__ void map_row(const MapArgs &a, int i, int b, int j, int slot, int len) {
    const int pos = len + j, page = a.table[(size_t)slot * a.max_blocks + pos / PAGE_POS];
    const bool mapped = a.last_live == nullptr || j <= a.last_live[b];
    a.slot_map[i] = mapped && (unsigned)page < (unsigned)a.n_pages ? page * PAGE_POS + pos % PAGE_POS : -1;      // (a free list that holds no page's number)
    a.row_pos[i] = pos;
}

template <int N>
__global__ __launch_bounds__(N) void map_pages_kernel(MapArgs a) {
    constexpr int NW = N / 64;
    __shared__ MapSums part[NW];
    __shared__ unsigned listed[MAP_MAX_SLOTS / 32];
    __shared__ MapTile<N> tile;
    __shared__ int bad, many;
    const int t = threadIdx.x;
    const int top = *a.n_free;
    const auto load = [&](int b) {
        MapSeq s{-1, 0, 0, 0, 0};
        if (b >= a.n_seqs) return s;
        s.rows = a.rows[b];
        s.slot = a.slots ? a.slots[b] : b;
        if ((unsigned)s.slot >= (unsigned)a.n_slots) { s.slot = -2; return s; }
        s.len = a.lens[s.slot];
        s.own = a.owned[s.slot];
        s.need = (int)(((long long)s.len + s.rows + PAGE_POS - 1) / PAGE_POS);
        return s;
    };
    const auto sums_of = [](const MapSeq &s) { return MapSums{s.own > s.need ? s.own - s.need : 0, s.need > s.own ? s.need - s.own : 0, s.rows}; };
    MapSeq mine = load(t);                                       // of the first tile, which is all there is up to N sequences
    if (t == 0) bad = many = 0;
    if (a.slots)
        for (int w = t; w < (a.n_slots + 31) / 32; w += N) listed[w] = 0;
    __syncthreads();
    // ---- what the lists ask for, and whether they make sense
    MapSums at_mine{}, sum_mine{};
    long long back = 0, more = 0, rows = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += N) {
        MapSeq s = b0 == 0 ? mine : load(b0 + t);
        int code = 0;
        if (s.slot == -2) code = LLMA_E_RANGE;
        else if (s.slot >= 0) {
            const bool twice = a.slots && (atomicOr(&listed[s.slot / 32], 1u << (s.slot % 32)) >> (s.slot % 32) & 1);
            if (twice || s.len < 0 || s.rows < 0 || s.own < 0 || s.own > a.max_blocks) code = LLMA_E_INVAL;
            else if (((long long)s.len + s.rows + PAGE_POS - 1) / PAGE_POS > a.max_blocks) code = LLMA_E_RANGE;
        }
        if (code) { atomicMin(&bad, code); s.own = s.need = s.rows = 0; }
        if (s.rows > 1 << 20 || s.own > 1 << 20 || s.need > 1 << 20) many = 1;       // (1024 of them may pass 32 bits)
        MapSums sum;
        const MapSums at = block_scan3<NW>(sums_of(s), part, &sum);
        back += sum.back; more += sum.more; rows += sum.rows;
        if (b0 == 0) { at_mine = at; sum_mine = sum; }
    }
    __syncthreads();
    // Rare: all of them once more, in pieces of 20 bits.  (Where the step is granted, the tiles' sums of pages are right: no more than 2^26 go back or are taken, so
    // none of them had passed 32 bits)
    if (many) {
        back = more = rows = 0;
        for (int b0 = 0; b0 < a.n_seqs; b0 += N) {
            const MapSeq s = b0 == 0 ? mine : load(b0 + t);
            const MapSums v = s.slot >= 0 ? sums_of(s) : MapSums{0, 0, 0};       // (of lists that make no sense: not used)
            MapSums low, high;
            (void)block_scan3<NW>(MapSums{v.back & 0xfffff, v.more & 0xfffff, v.rows & 0xfffff}, part, &low);
            (void)block_scan3<NW>(MapSums{v.back >> 20, v.more >> 20, v.rows >> 20}, part, &high);
            back += low.back + ((long long)high.back << 20);
            more += low.more + ((long long)high.more << 20);
            rows += low.rows + ((long long)high.rows << 20);
        }
        __syncthreads();
    }
    int status = bad;
    if (status == 0 && (top < 0 || back > a.n_pages || top > a.n_pages - (int)back)) status = LLMA_E_INVAL;
    // (without a slot map only the tables and offsets are wanted: any number of rows)
    if (status == 0 && (rows > 0x7fffffffll || (a.max_rows > 0 && rows > a.max_rows))) status = LLMA_E_RANGE;
    const int stack = top + (status == 0 ? (int)back : 0);       // its height once everything is back
    if (status == 0 && more > stack) status = (int)(more - stack < 0x7fffffff ? more - stack : 0x7fffffff);
    const bool ok = status == 0, here = a.max_rows > 0 && a.max_rows <= MAP_ROWS_HERE;      // (no map: no row has a place in one)
    if (t == 0) *a.status = status;
    // a tile's sequences and their places, for threads that look them up by page or row
    const auto look = [&](int b0, MapSums *at, MapSums *sum) {
        const MapSeq s = b0 == 0 ? mine : load(b0 + t);
        if (b0 == 0) { *at = at_mine; *sum = sum_mine; }
        else *at = block_scan3<NW>(sums_of(s), part, sum);
        __syncthreads();
        tile.seq[t] = s;
        return s;
    };
    if (ok && back > 0) {
        // ---- pages that go back: the j-th of them in granting order lies j below the stack's new top
        int before = 0;
        for (int b0 = 0; b0 < a.n_seqs; b0 += N) {
            MapSums at, sum;
            (void)look(b0, &at, &sum);
            tile.first[t] = at.back;
            __syncthreads();
            for (int i = t; i < sum.back; i += N) {
                const int q = count_le(tile.first, N, i) - 1;
                int *entry = a.table + (size_t)tile.seq[q].slot * a.max_blocks + tile.seq[q].need + (i - tile.first[q]);
                a.free_pages[stack - 1 - (before + i)] = *entry;
                *entry = -1;
            }
            before += sum.back;
        }
        __syncthreads();
    }
    // ---- pages that are granted, and the rows
    int granted = 0, row0 = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += N) {
        MapSums at, sum;
        const MapSeq s = look(b0, &at, &sum);
        if (!ok) at = sum = MapSums{0, 0, 0};
        if (b0 + t < a.n_seqs) {
            a.row_offsets[b0 + t] = row0 + at.rows;
            a.lens_after[b0 + t] = s.len + (ok ? s.rows : 0);
        }
        if (sum.more > 0) {                                      // (uniform)
            tile.first[t] = at.more;
            __syncthreads();
            for (int i = t; i < sum.more; i += N) {
                const int q = count_le(tile.first, N, i) - 1;
                a.table[(size_t)tile.seq[q].slot * a.max_blocks + tile.seq[q].own + (i - tile.first[q])] = a.free_pages[stack - 1 - (granted + i)];
            }
            granted += sum.more;
            __syncthreads();
        }
        if (ok && s.slot >= 0) a.owned[s.slot] = s.need;
        if (here && sum.rows > 0) {
            tile.first[t] = at.rows;
            __syncthreads();
            for (int i = t; i < sum.rows; i += N) {
                const int q = count_le(tile.first, N, i) - 1;
                map_row(a, row0 + i, b0 + q, i - tile.first[q], tile.seq[q].slot, tile.seq[q].len);
            }
        }
        row0 += sum.rows;
    }
    if (t == 0) {
        a.row_offsets[a.n_seqs] = row0;
        if (ok) *a.n_free = stack - granted;
    }
    if (here)
        for (int i = row0 + t; i < a.max_rows; i += N) { a.slot_map[i] = -1; a.row_pos[i] = 0; }
}
#define MAP_OFFSETS 8192         // sequences whose offsets a workgroup of map_rows_kernel keeps in LDS
__global__ __launch_bounds__(256) void map_rows_kernel(MapArgs a) {
    __shared__ int offsets[MAP_OFFSETS + 1];
    const bool kept = a.n_seqs <= MAP_OFFSETS;
    if (kept)
        for (int b = threadIdx.x; b <= a.n_seqs; b += 256) offsets[b] = a.row_offsets[b];
    __syncthreads();
    const int total = kept ? offsets[a.n_seqs] : a.row_offsets[a.n_seqs];
    for (int i = blockIdx.x * 512 + threadIdx.x; i < a.max_rows && i < (int)(blockIdx.x + 1) * 512; i += 256) {
        if (i >= total) {
            a.slot_map[i] = -1;
            a.row_pos[i] = 0;
            continue;
        }
        const int b = kept ? count_le(offsets + 1, a.n_seqs, i) : count_le(a.row_offsets + 1, a.n_seqs, i), slot = a.slots ? a.slots[b] : b;
        map_row(a, i, b, i - (kept ? offsets[b] : a.row_offsets[b]), slot, a.lens[slot]);
    }
}
void launch_map_pages(const MapArgs &a, hipStream_t st) {
    // (a step of a few sequences: four waves wait for each other sooner than sixteen)
    if (a.n_seqs <= 256 && a.max_rows <= 2048) hipLaunchKernelGGL(map_pages_kernel<256>, dim3(1), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(map_pages_kernel<MAP_THREADS>, dim3(1), dim3(MAP_THREADS), 0, st, a);
    if (a.max_rows > MAP_ROWS_HERE) hipLaunchKernelGGL(map_rows_kernel, dim3((a.max_rows + 511) / 512), dim3(256), 0, st, a);
}

__global__ __launch_bounds__(256) void pass_rows_kernel(const PromptSeg *segs, const int *batch_slots, int n_seqs, int m, const int *last_live, int *rows, int *slots) {
    for (int b = threadIdx.x; b < n_seqs; b += 256) {
        rows[b] = segs ? segs[b].rows : last_live && n_seqs == 1 && *last_live + 1 < m ? *last_live + 1 : m;
        slots[b] = segs ? segs[b].slot : batch_slots[b];
    }
}
void launch_pass_rows(const PromptSeg *segs, const int *batch_slots, int n_seqs, int m, const int *last_live, int *rows, int *slots, hipStream_t st) {
    hipLaunchKernelGGL(pass_rows_kernel, dim3(1), dim3(256), 0, st, segs, batch_slots, n_seqs, m, last_live, rows, slots);
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

// ---------------------------------------------------------------------------------------------
// write into the cache
// ---------------------------------------------------------------------------------------------
// A run = rows with consecutive slots inside one page.  Per run and head: the smallest power of two s with max |x| / s <= 448 (over finite
// values); a run that starts inside its page keeps the page's scale where that is larger, and where s is larger the
// codes before it are rounded again to the new scale.  code = x / s rounded to nearest even: the division is exact, so the one rounding
// to four significant bits is the format's.  +-inf become +-448, NaN stays NaN.
// 16 (8) lanes share a row's 128 (64) features, eight each, and a lane has four neighbouring positions, so that a dim's four codes leave as one word
// of the transposed V: a wave holds 16 (32) positions.  A prompt's pages take a wave for each 16 (32) positions, which agree on the maximum in LDS; a step's
// runs, a few rows long, one wave.
// Prompts are bound by memory: 4 of up to 2011 fp32 rows of 8 heads of 128, 62 MB read and written, 17 us = 3.6 TB/s.  Steps by their chain of slots, rows, maximum and
// scale: 16 sequences of 9 rows of 32 heads 9.5 us, a single one 5.8; keeping two rounds of rows from the maximum to the codes
// made runs of 17 rows faster (8.4 to 7.5) and those of nine slower (5.9 to 6.5).
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// exponent of the scale: -64 .. 120
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);      // 448 = 1.75 * 2^8
    return e < -64 ? -64 : e > 120 ? 120 : e;
}
__device__ __forceinline__ float code_input(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_input(a), code_input(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_input(c), code_input(d), (int)w, true);
}
// four codes' values times `by`, as codes
__device__ __forceinline__ uint32_t codes_by(uint32_t c, float by) {
    return codes4(__builtin_amdgcn_cvt_f32_fp8((int)c, 0) * by, __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * by, __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * by, __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * by);
}

template <int DH, int TYPE, bool KEYS, int WAVES>
__device__ __forceinline__ void append_run(const AppendArgs &a, int head, int row0, int n, int page, int off, float *shared_max) {
    constexpr int LPR = DH / 8;                     // lanes per row
    constexpr int QUADS = 64 / LPR;                 // groups of four positions a wave has at once
    const int lane = threadIdx.x & 63, wave = WAVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int d0 = lane % LPR * 8;
    const size_t block = (size_t)page * a.c.heads + head;
    uint8_t *const codes = (KEYS ? a.c.k : a.c.v) + block * (PAGE_POS * DH);
    float *const scale = (KEYS ? a.c.k_scale : a.c.v_scale) + block;
    const float old = off > 0 ? *scale : 0.f;
    const void *const src = KEYS ? a.k : a.v;
    const int64_t rs = KEYS ? a.k_row : a.v_row, hs = KEYS ? a.k_head : a.v_head;
    const int quad0 = off / 4, rounds = ((off + n - 1) / 4 - quad0) / QUADS + 1;      // (the run's groups, QUADS a round)
    float x[4][8];
    const auto load = [&](int r) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = 4 * (quad0 + r * QUADS + lane / LPR) + j - off;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[j][e] = 0.f;
            if (i < 0 || i >= n) continue;
            if constexpr (TYPE == ROWS_TILED) {
                const bf16_t *p = (const bf16_t *)src + head * hs;
                if constexpr (KEYS) {
                    row8<ROWS_BF16>(p, (int64_t)kcache_off(row0 + i, d0, DH), x[j]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[j][e] = bf16_to_f32(p[vcache_off(row0 + i, d0 + e, DH)]);
                }
            } else {
                row8<TYPE>(src, (int64_t)(row0 + i) * rs + head * hs + d0, x[j]);
            }
        }
    };
    float amax = 0.f;
    for (int r = wave; r < rounds; r += WAVES) {
        load(r);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float m = fabsf(x[j][e]);
                amax = m < __builtin_huge_valf() ? fmaxf(amax, m) : amax;          // (false for NaN)
            }
    }
    butterfly<32>([&](auto o) { amax = fmaxf(amax, lane_xor<o.value>(amax)); });
    if constexpr (WAVES > 1) {
        __syncthreads();                            // (the last run's maxima have been read)
        if (lane == 0) shared_max[wave] = amax;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) amax = fmaxf(amax, shared_max[w]);
    }
    float s = pow2(scale_exponent(amax));
    if (off > 0) {
        if (s > old) {
            // The codes before the run, 16 bytes a lane and four of them at once: off rows of K, the first off bytes of V's rows, where 16 bytes that the run begins
            // in are written byte by byte (another wave may be writing its positions).  By single bytes a step into 32
            // heads' pages of 60 positions that all had to grow took 22 us more than one into pages that had not; so 4
            const float by = old / s;
            const int per = KEYS ? 1 : (off + 15) / 16, pieces = KEYS ? off * DH / 16 : DH * per;
            for (int i0 = wave * 64 + lane; i0 < pieces; i0 += 4 * 64 * WAVES) {
                u32x4 c[4];
                u32x4 *at[4];
                int mine[4];                        // bytes before the run
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + u * 64 * WAVES;
                    const int piece = i < pieces ? i : i0;
                    at[u] = (u32x4 *)(KEYS ? codes + piece * 16 : codes + piece / per * PAGE_POS + piece % per * 16);
                    mine[u] = i >= pieces ? 0 : KEYS ? 16 : off - piece % per * 16;
                    c[u] = *at[u];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) c[u][w] = codes_by(c[u][w], by);
                    if (mine[u] >= 16) {
                        *at[u] = c[u];
                    } else {
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            if (mine[u] >= 4 * w + 4) {
                                ((uint32_t *)at[u])[w] = c[u][w];
                                continue;
                            }
#pragma unroll
                            for (int e = 0; e < 3; ++e)
                                if (4 * w + e < mine[u]) ((uint8_t *)at[u])[4 * w + e] = (uint8_t)(c[u][w] >> 8 * e);
                        }
                    }
                }
            }
        } else {
            s = old;
        }
    }
    if (wave == 0 && lane == 0) *scale = s;
    const float inv = 1.f / s;                      // (exact)
    for (int r = wave; r < rounds; r += WAVES) {
        if (rounds > WAVES) load(r);                // (a wave with several rounds has kept none)
        const int p0 = 4 * (quad0 + r * QUADS + lane / LPR);     // the lane's positions in the page
        if (p0 + 3 < off || p0 >= off + n) continue;
        uint32_t w[4][2];                           // [position]: eight dims' codes
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float *v = x[j];
            w[j][0] = codes4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            w[j][1] = codes4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
        }
        if constexpr (KEYS) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (p0 + j >= off && p0 + j < off + n) *(u32x2 *)(codes + (p0 + j) * DH + d0) = (u32x2){w[j][0], w[j][1]};
        } else {
            const bool whole = p0 >= off && p0 + 3 < off + n;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int sh = e % 4 * 8;
                uint8_t *const to = codes + (d0 + e) * PAGE_POS + p0;
                if (whole) {
                    *(uint32_t *)to = (w[0][e / 4] >> sh & 255) | (w[1][e / 4] >> sh & 255) << 8 | (w[2][e / 4] >> sh & 255) << 16 | (w[3][e / 4] >> sh) << 24;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (p0 + j >= off && p0 + j < off + n) to[j] = (uint8_t)(w[j][e / 4] >> sh);
                }
            }
        }
    }
}

// WAVES waves (WAVES > 1: a workgroup) per window of rows, head, and K or V: the runs that begin in the window, one after the other
template <int DH, int TYPE, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void append_paged_kernel(AppendArgs a, int window, int n_windows) {
    __shared__ float shared_max[WAVES];
    const int unit = WAVES == 1 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
    const int lane = threadIdx.x & 63;
    const int win = unit / (2 * a.c.heads), head = unit % (2 * a.c.heads) / 2;
    if (win >= n_windows) return;
    const int r0 = win * window;
    // the slots of the window and of the rows a run from it can reach; which of them go on from the row before
    const auto slot_of = [&](int i) { return i >= 0 && i < a.n_rows ? a.slot_map[i] : -1; };
    const int slot = slot_of(r0 + lane), behind = slot_of(r0 + 64 + lane);
    int prev = __shfl_up(slot, 1), prev_behind = __shfl_up(behind, 1);
    const int before = slot_of(r0 - 1), last = __builtin_amdgcn_readlane(slot, 63);
    if (lane == 0) { prev = before; prev_behind = last; }
    const auto goes_on = [&](int s, int p) { return p >= 0 && s == p + 1 && s % PAGE_POS != 0; };
    const unsigned long long on = __ballot(goes_on(slot, prev)), on_behind = __ballot(goes_on(behind, prev_behind));
    unsigned long long begins = __ballot(lane < window && slot >= 0 && slot / PAGE_POS < a.c.n_pages) & ~on;
    int turn = 0;
    while (begins) {
        const int at = __builtin_ctzll(begins);
        begins &= begins - 1;
        const int first = __builtin_amdgcn_readlane(slot, at), off = first % PAGE_POS;
        // its length: the rows that go on, 64 at most
        const unsigned long long rest = at == 63 ? on_behind : (on >> (at + 1)) | (on_behind << (63 - at));
        const int n = ~rest == 0 ? 64 : __builtin_ctzll(~rest) + 1;
        if constexpr (WAVES > 1) {
            // A run that one wave holds goes to one of them, in turn, the longer ones to all together: 64 sequences of 9 rows x 32 heads 52 -> 23 us, 200 of 5
            // 79 -> 36; windows of 32 rows 18 and 35, but for 4 prompts of 2011 rows x 8 heads 18 -> 21
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quads = (off + n - 1) / 4 - off / 4 + 1;
            if (quads <= 512 / DH) {
                if (turn++ % WAVES != wave) continue;
                if (unit & 1) append_run<DH, TYPE, false, 1>(a, head, r0 + at, n, first / PAGE_POS, off, shared_max);
                else append_run<DH, TYPE, true, 1>(a, head, r0 + at, n, first / PAGE_POS, off, shared_max);
                continue;
            }
        }
        if (unit & 1) append_run<DH, TYPE, false, WAVES>(a, head, r0 + at, n, first / PAGE_POS, off, shared_max);
        else append_run<DH, TYPE, true, WAVES>(a, head, r0 + at, n, first / PAGE_POS, off, shared_max);
    }
}

void launch_append_paged(const AppendArgs &a, hipStream_t st) {
    if (a.n_rows < 1) return;
    // Windows of 64 rows (a prompt's pages) as long as they give the chip its waves, with all of a page's waves at work; else windows so small that there are
    // enough of them, a wave each: a step's runs are short.
    const int units = 2 * a.c.heads, waves = a.c.dh == 128 ? 4 : 2;
    const bool pages = (int64_t)((a.n_rows + 63) / 64) * units * waves >= 2048;
    int window = 64;
    while (!pages && window > 1 && (int64_t)((a.n_rows + window - 1) / window) * units < 4096) window /= 2;
    const int n_windows = (a.n_rows + window - 1) / window;
    const int64_t n = (int64_t)n_windows * units;
    auto of = [&](auto dh, auto type) {
        constexpr int DH = decltype(dh)::value, TYPE = decltype(type)::value, W = DH == 128 ? 4 : 2;
        if (pages) hipLaunchKernelGGL((append_paged_kernel<DH, TYPE, W>), dim3((unsigned)n), dim3(64 * W), 0, st, a, window, n_windows);
        else hipLaunchKernelGGL((append_paged_kernel<DH, TYPE, 1>), dim3((unsigned)((n + 3) / 4)), dim3(256), 0, st, a, window, n_windows);
    };
    auto typed = [&](auto dh) {
        if (a.type == ROWS_BF16) of(dh, std::integral_constant<int, ROWS_BF16>{});
        else if (a.type == ROWS_F16) of(dh, std::integral_constant<int, ROWS_F16>{});
        else if (a.type == ROWS_F32) of(dh, std::integral_constant<int, ROWS_F32>{});
        else of(dh, std::integral_constant<int, ROWS_TILED>{});
    };
    if (a.c.dh == 128) typed(std::integral_constant<int, 128>{});
    else typed(std::integral_constant<int, 64>{});
}

// ---------------------------------------------------------------------------------------------
// attention over the pages
// ---------------------------------------------------------------------------------------------
// Row j of sequence b sees positions 0 .. len - rows + j.  A key head's query rows (rows x query heads per key head) are the columns
// of both products: S^T = K Q^T, O^T = V^T P^T, 16 rows a tile, NT tiles a wave.  Row i of score tile g is position 16 (i/4) + 4 g + i%4 of the page,
// so that a lane's 16 probabilities are those of 16 neighbouring positions -- the ones its V bytes hold.
// One pass with the running maximum and sum of the softmax in fp32; scores in powers of two.
// The pages of all sequences, end to end, are cut into equal shares, one per workgroup and key head: ragged lengths load the chip
// evenly, and a share's four waves take its pages in turn and meet in LDS at a sequence's end.  A sequence that lies in one share
// is finished there; the others' parts are joined by attend_join_kernel.
// Steps are bound by one read of the cache: 16 sequences of up to 4096 positions, 9 rows of 32 heads of 128, 361 MB in 76 to 83 us a call = 4.4 to 4.7 TB/s, 61 of 5 rows, four
// query heads a key head, fp16, 671 MB in 148 to 155 = 4.3 to 4.5.  This kernel alone takes 79 and 148 us under the profiler, one of the same mapping that only loads 75 and 130.
// Short sequences are not cut: a workgroup per sequence and key head, no count of the others' pages, nothing to join.  It is bound by what one compute unit
// takes in, 44 KB a microsecond, so it pays while a table's row holds few pages more than an equal share would.  us inside a captured graph, cut and whole, 9 rows of 32 heads of 128:
//                     1 x 512    1 x 1001   1 x 1500   6 x 1001   6 x 2000   16 x 512   16 x 1001  64 x 1001  64 x 1900
//   bf16              11.5 10.5  12.0 11.9  12.5 14.5  20.7 13.6  27.5 20.4  24.5 17.1  30.0 22.0  85.3 81.4  153 150
//   fp16              11.5 11.1  12.3 12.7  12.7 15.8  21.1 14.4  27.8 22.0  25.7 17.8  31.0 23.0  88.9 84.0  154 152
//   fp32              11.9 11.7  12.6 13.5  13.1 17.0  22.2 15.3  29.0 23.4  26.1 18.9  32.1 23.4  91.8 91.2  160 161
// and a bf16 call of its own, 64 of 3900 256 and 262, four of 5 rows, 8 key heads, 1001 / 2000 13.5 / 13.2 and 11.2 / 16.6.  Eight waves for one compute unit instead of four changed nothing.
#define ATTEND_CUS 256           // compute units; two workgroups each, one where three or four tiles fill the registers
#define ATTEND_MIN_PAGES 4       // of a share: a page per wave

#define ATTEND_WHOLE_PAGES 40    // whole sequences: of a table's row, at most
struct AttendPlan { int nt, tiles, shares; bool whole; };        // whole: sequences in place of shares
static AttendPlan attend_plan(int n_seqs, int max_blocks, int n_heads, int kv_heads, int dh, int max_rows) {
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
    const int64_t beyond = (max_blocks - pages * columns / groups) * dh;
    p.whole = max_blocks <= ATTEND_WHOLE_PAGES && n_seqs * columns < 1 << 23 && beyond <= 128 * (n_seqs * columns >= ATTEND_CUS / 2 ? 32 : n_seqs > 1 ? 16 : 12);
    return p;
}
// work: [pages before every sequence, n_seqs + 1 ints, rounded up to 64][parts' O][parts' m][parts' l].  (Also where sequences stay whole: a workspace
// for some number of sequences does for fewer)
__host__ __device__ static inline int64_t attend_parts(const AttendPlan &p, int kv_heads) { return p.shares > 1 ? (int64_t)p.shares * 2 * kv_heads * p.tiles : 0; }
int64_t attend_paged_bytes(int n_seqs, int max_blocks, int n_heads, int kv_heads, int dh, int max_rows) {
    const AttendPlan p = attend_plan(n_seqs, max_blocks, n_heads, kv_heads, dh, max_rows);
    return ((int64_t)(n_seqs + 1 + 63) / 64 * 64 + attend_parts(p, kv_heads) * 16 * p.nt * (dh + 2)) * 4;
}

struct AttendSeq { int slot, len, rows, row0, seen; };          // seen: the last position that its first row sees
// a sequence as the kernels take it: whatever the lists hold, nothing outside the buffers is reached
__device__ __forceinline__ AttendSeq attend_seq(const AttendArgs &a, int b) {
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
template <int DH, int NT, int TYPE>
__device__ __forceinline__ void attend_load_q(const AttendArgs &a, const AttendSeq &s, int head, int group, int r0, AttendQ<DH, NT> &q) {
#pragma unroll
    for (int u = 0; u < (attend_pieces<DH, NT> + 255) / 256; ++u) {
        const int i = u * 256 + threadIdx.x, lane = i & 63, half = i >> 6 & 1, t = (i >> 7) % (DH / 64), nt = (i >> 7) / (DH / 64);
        const int r = r0 + nt * 16 + (lane & 15), d = 64 * t + 16 * (lane >> 4) + 8 * half;
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
// 16 codes as two operands of eight bf16, times a power of two
__device__ __forceinline__ void widen16(u32x4 c, float scale, u32x4 &lo, u32x4 &hi) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        lo[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w], scale, false));
        lo[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w], scale, true));
        hi[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 + w], scale, false));
        hi[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 + w], scale, true));
    }
}
// the same as fp16, and their product
__device__ __forceinline__ void widen16_half(u32x4 c, float scale, u32x4 &lo, u32x4 &hi) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        lo[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[w], scale, false));
        lo[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[w], scale, true));
        hi[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 + w], scale, false));
        hi[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 + w], scale, true));
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
// fp16 products keep their sums in units of a power of two, `now` its exponent as fp32 holds it, so that V fits: a code of 2^-9 .. 448 times 2^-15 .. 2^7 is exact in fp16.
// A page whose scale is not that near the unit makes its own the unit, but none more than 2^60 below the largest before it (up to 2^62 units may have been
// added up, and fp32 ends at 2^128): there V counts as zero where it is more than 2^75 below another page's.
struct SumUnit { int now, least; };
// What a page's codes are multiplied by (a scale of 0 is no page's: its codes are 0, and the unit stays); the sums have to follow the unit.  (Without branches: 272 us for
// two sequences of up to 2047 rows, 275 with one; 267 where the unit never changes.)
__device__ __forceinline__ float unit_factor(float scale, SumUnit &u) {
    const int e = (int)(__float_as_uint(scale) >> 23 & 255), near = e > u.least ? e : u.least;
    const bool other = ((unsigned)(e - u.now + 15) > 22u) & (e > 0);
    u.now = other ? near : u.now;
    u.least = u.now - 60 > u.least ? u.now - 60 : u.least;
    return pow2(e - u.now > -126 ? e - u.now : -126);
}
__device__ __forceinline__ f32x4 times_pow2(f32x4 v, int e) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = __builtin_amdgcn_ldexpf(v[r], e);
    return v;
}
// the NaN codes among four: 0x80 in their bytes
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t whole_bytes(uint32_t m) { return m | (m - (m >> 7)); }
// a word's first n bytes (all for n >= 4, none for n <= 0)
__device__ __forceinline__ uint32_t bytes_below(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : ~(~0u << (8 * n)); }
// four such bytes as the ones of two words of bf16
__device__ __forceinline__ u32x2 ones_of(uint32_t m) { return (u32x2){(m >> 7 & 1) * 0x3f80u | (m >> 15 & 1) * 0x3f800000u, (m >> 23 & 1) * 0x3f80u | (m >> 31) * 0x3f800000u}; }

// rare: a page's V holds NaN where not all rows see it.  The rows that see one get it in that feature; products of ones find them.  codes: the page's V at the lane's place
template <int DH, int NT>
__device__ __forceinline__ void attend_nans(const uint8_t *codes, int base, int len, const int (&limit)[NT], f32x4 (&o)[NT][DH / 16]) {
    const int kb = (threadIdx.x & 63) >> 4;
#pragma unroll 1
    for (int d = 0; d < DH / 16; ++d) {
        const u32x4 c = *(const u32x4 *)(codes + 16 * d * PAGE_POS);
        u32x4 ones[2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const u32x2 o2 = ones_of(nan_bytes(c[w] & bytes_below(len - base - 16 * kb - 4 * w)));
            ones[w / 2][2 * (w & 1)] = o2[0];
            ones[w / 2][2 * (w & 1) + 1] = o2[1];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            f32x4 hit = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 sees;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int p = base + 16 * kb + 8 * u + 2 * w;
                    sees[w] = (p <= limit[n] ? 0x3f80u : 0) | (p + 1 <= limit[n] ? 0x3f800000u : 0);
                }
                hit = mfma16x16x32(ones[u], sees, hit);
            }
#pragma unroll
            for (int e = 0; e < DH / 16; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (e == d && hit[r] > 0.f) o[n][e][r] = __builtin_nanf("");
        }
    }
}

template <int TYPE>
__device__ __forceinline__ void attend_store(const AttendArgs &a, int row, int h, int d, f32x4 v) {      // four neighbouring features
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

template <int DH, int NT, int TYPE> constexpr int attend_lds = 16 * (attend_nq<TYPE> * attend_pieces<DH, NT> > 4 * NT * (DH / 16) * 64 ? attend_nq<TYPE> * attend_pieces<DH, NT> : 4 * NT * (DH / 16) * 64);
#define ATTEND_KEPT 256          // sequences whose lengths and rows the workgroup keeps in LDS

template <int DH, int NT, int TYPE>
__global__ __launch_bounds__(256, NT <= 2 ? 2 : 1) void attend_paged_kernel(AttendArgs a, AttendPlan plan) {
    constexpr bool HALF = TYPE == ROWS_BF16 && NT > 2;
    constexpr float BIAS = HALF ? 15.f : 0.f;
    constexpr int NQ = attend_nq<TYPE>, NP = attend_np<TYPE, HALF>;
    constexpr int TD = DH / 64, DT = DH / 16, PIECES = attend_pieces<DH, NT>;
    extern __shared__ u32x4 lds[];
    u32x4 *const q = lds;
    f32x4 *const osum = (f32x4 *)lds;                            // the four waves' sums, in the queries' place once they are used
    __shared__ float ml[4][2][NT * 16];
    __shared__ int part[4];
    __shared__ AttendSeq kept[ATTEND_KEPT];
    int *const starts = (int *)((char *)lds + attend_lds<DH, NT, TYPE>);         // [n_seqs + 1]
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
    const float to_log2 = a.scale * 1.44269504088896340736f;
    const int kb = lane >> 4, col = lane & 15;
    const uint32_t k_off = (16 * (col >> 2) + (col & 3)) * DH + 16 * kb, v_off = col * PAGE_POS + 16 * kb;

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
    u32x4 kc[4][TD], vc[DT];
    const auto block_of = [&](int page) { return ((size_t)(page < 0 ? 0 : page) * a.c.heads + head) * (PAGE_POS * DH); };
    const auto take_k = [&](size_t block) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int t = 0; t < TD; ++t) kc[g][t] = *(const u32x4 *)((a.c.k + block + 4 * g * DH + 64 * t) + k_off);
    };
    const auto take_v = [&](size_t block, int d) { vc[d] = *(const u32x4 *)((a.c.v + block + 16 * d * PAGE_POS) + v_off); };
    const auto take_page = [&](int page) {
        take_k(block_of(page));
#pragma unroll
        for (int d = 0; d < DT; ++d) take_v(block_of(page), d);
    };
    float ks = 0.f, vs = 0.f;
    const auto take_scales = [&](int id) {
        ks = vs = 0.f;
        if (id >= 0) {
            ks = a.c.k_scale[(size_t)id * a.c.heads + head];
            vs = a.c.v_scale[(size_t)id * a.c.heads + head];
        }
    };

    AttendSeg seg = segment(uniform(count_le(starts, n_seqs + 1, p0) - 1));
    AttendQ<DH, NT> qr;
    int id = -1;
    if (seg.last > 0) {
        id = page_ids(seg, seg.first + wave);
        attend_load_q<DH, NT, TYPE>(a, seg.s, head, group, r0, qr);
        if (seg.first + wave < seg.last) take_page(__builtin_amdgcn_readlane(id, 0));
        take_scales(id);
    }
    while (seg.last > 0) {
        const AttendSeq s = seg.s;
        __syncthreads();
        attend_put_q<DH, NT, NQ, TYPE>(qr, q);
        __syncthreads();
        const AttendSeg after = segment(seg.b + 1);
        int id_after = -1;
        if (after.last > 0) {
            id_after = page_ids(after, after.first + wave);
            attend_load_q<DH, NT, TYPE>(a, after.s, head, group, r0, qr);
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
        SumUnit unit{127, 67};
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
                const float pks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), it)), pvs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), it));
                const size_t next = block_of(__builtin_amdgcn_readlane(id, it + 1 < n_here ? it + 1 : it));      // (the last page's once more: no branch around the loads)
                // (several tiles' queries come from LDS for every page: kept in registers across pages they would push the sums out)
                int ql = lane;
                if constexpr (NT > 1) asm volatile("" : "+v"(ql));
                f32x4 sc[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int g = 0; g < 4; ++g) sc[n][g] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < TD; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        u32x4 lo, hi;
                        widen16(kc[g][t], 1.f, lo, hi);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int pl = NQ - 1; pl >= 0; --pl) {
                                sc[n][g] = mfma16x16x32(lo, q[pl * PIECES + ((n * TD + t) * 2) * 64 + ql], sc[n][g]);
                                sc[n][g] = mfma16x16x32(hi, q[pl * PIECES + ((n * TD + t) * 2 + 1) * 64 + ql], sc[n][g]);
                            }
                    }
                __builtin_amdgcn_sched_barrier(0);
                take_k(next);
                __builtin_amdgcn_sched_barrier(0);
                const float by = to_log2 * pks;
                const bool masked = page < 0 || base + PAGE_POS - 1 > seen;
                uint32_t nans = 0;
                if (masked) {
                    const int there = page < 0 ? 0 : s.len - base - 16 * kb;       // of the lane's 16 positions of V
                    uint32_t is[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) is[w] = bytes_below(there - 4 * w);
                    // what lies behind the last position may be anything, and a NaN that only later rows see must not reach the others through 0 * NaN
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t c = vc[d][w] & is[w], m = nan_bytes(c);
                            nans |= m;
                            vc[d][w] = c & ~whole_bytes(m);
                        }
                }
                u32x4 pb[NT][NP][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float x[16], top = LLMA_NEG_INF;
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = sc[n][e / 4][e % 4] * by;
                    if (masked) {
                        const int left = (page < 0 ? -1 : limit[n]) - base - 16 * kb;
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = e > left ? LLMA_NEG_INF : x[e];
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, x[e]);
                    top = fmaxf(top, lane_xor<16>(top));
                    top = fmaxf(top, lane_xor<32>(top));
                    const float mn = fmaxf(m[n], top), ref = mn == LLMA_NEG_INF ? 0.f : mn, from = ref - BIAS;
                    const float keep = __builtin_amdgcn_exp2f(m[n] - ref);
                    m[n] = mn;
                    l[n] *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] *= keep;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e] = __builtin_amdgcn_exp2f(x[e] - from);
                        l[n] += x[e];
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            float y = x[8 * u + 2 * w], z = x[8 * u + 2 * w + 1];
#pragma unroll
                            for (int pl = 0; pl < NP; ++pl) {
                                pb[n][pl][u][w] = HALF ? half_pair(y, z) : bf16_pair(y, z);
                                if (pl + 1 < NP) { y -= __uint_as_float(pb[n][pl][u][w] << 16); z -= __uint_as_float(pb[n][pl][u][w] & 0xffff0000u); }
                            }
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (masked && __ballot(nans != 0) != 0) attend_nans<DH, NT>(a.c.v + block_of(page) + v_off, base, s.len, limit, o);
                float v_by = pvs;
                if constexpr (HALF) {
                    const int was = unit.now;
                    v_by = unit_factor(pvs, unit);
                    if (unit.now != was) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int d = 0; d < DT; ++d) o[n][d] = times_pow2(o[n][d], was - unit.now);
                    }
                }
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    u32x4 lo, hi;
                    if constexpr (HALF) widen16_half(vc[d], v_by, lo, hi);
                    else widen16(vc[d], v_by, lo, hi);
                    take_v(next, d);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int pl = NP - 1; pl >= 0; --pl) {
                            o[n][d] = HALF ? mfma16x16x32_half(lo, pb[n][pl][0], o[n][d]) : mfma16x16x32(lo, pb[n][pl][0], o[n][d]);
                            o[n][d] = HALF ? mfma16x16x32_half(hi, pb[n][pl][1], o[n][d]) : mfma16x16x32(hi, pb[n][pl][1], o[n][d]);
                        }
                }
            }
            if (i0 + 256 < stop) {                               // (a share of more than 256 pages of one sequence)
                id = page_ids(seg, i0 + 256);
                take_page(__builtin_amdgcn_readlane(id, 0));
                take_scales(id);
            }
        }
        id = id_after;
        if (after.last > 0) {
            if (after.first + wave < after.last) take_page(__builtin_amdgcn_readlane(id, 0));
            take_scales(id);
        }
        // ---- the waves' sums meet
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] += lane_xor<16>(l[n]);
            l[n] += lane_xor<32>(l[n]);
            if constexpr (HALF) l[n] *= pow2(-15);
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
            for (int d = 0; d < DT; ++d) osum[((wave * NT + n) * DT + d) * 64 + lane] = HALF ? times_pow2(o[n][d] * f, unit.now - 127 - 15) : o[n][d] * f;
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
                const int d = 4 * u + wave;
                f32x4 v = osum[(n * DT + d) * 64 + lane];
#pragma unroll
                for (int w = 1; w < 4; ++w) v += osum[((w * NT + n) * DT + d) * 64 + lane];
                if (whole) attend_store<TYPE>(a, row, h, 16 * d + 4 * kb, v * inv);
                else *(f32x4 *)(po + (at * 16 * NT + 16 * n + col) * DH + 16 * d + 4 * kb) = v;
            }
            if (!whole && wave == 0 && kb == 0) { pm[at * 16 * NT + 16 * n + col] = top[n]; pl[at * 16 * NT + 16 * n + col] = sum[n]; }
        }
        seg = after;
    }
}

// ---- many rows -----------------------------------------------------------------------------------
// Which calls take it: those with more rows a key head than the shares' kernel holds (64) and at least this many row blocks.  Fewer leave compute units
// without work, where shares cut the pages too.  us inside a captured graph, here and in shares, 32 heads of 128, 1000 positions before 512 / 640 / 768 rows (128, 160, 192 blocks; fp32
// twice as many), 16 sequences of 18 x 4 rows over 4000 positions (128), 64 of 20 x 4 over 1000 (512):
//   bf16  47.6 33.4   50.1 60.0   54.7 62.3   107 75   43 90
//   fp16  62.2 43.6   65.3 78.8   71.1 81.6   142 96   57 117
//   fp32  49.4 60.1   59.8 104    64.8 106    114 126  71 157
// fp32 with 160 / 256 rows (96, 128 blocks) 38.9 / 42.0 and 45.2 / 46.9: its blocks would pay from fewer on.
#define ROWS_MIN 160
// Prompts: a workgroup takes 64 NT rows of a sequence's key head and all pages they see.  Each page is widened once, for all four waves, into LDS as the
// operands' images (16 KB of K, 16 KB of V at head_dim 128); a page is requested two ahead, widened one ahead, one barrier a page.  A wave holds its rows' queries and
// sums in registers and meets nobody at the end.  Pages behind a wave's rows are skipped; the longest row blocks start first, and a key head's on one XCD.
// The reference of the exponentials moves only when a maximum passes it by 2^8: the sums are rescaled once or twice a row instead of once a page.
// Bound by issue: two sequences of up to 2047 rows, 32 query and 8 key heads of 128, over up to 2900 positions before, bf16, 136 GFLOP in 272 us = 0.50 PFLOP/s, vector instructions
// in 46 % of the compute units' busy cycles, matrix instructions in 39 %, LDS in 28 %.  The exponentials of one page beside the products of the next spilled (330 to 430 us); eight waves a page, 256
// rows, 2 % faster there and 10 % slower for prompts without a cache (84 us against 76 for 2047 rows of 32 heads).
template <int DH> constexpr int rows_images = (4 * (DH / 64) * 2 + (DH / 16) * 2) * 64;       // 16-byte pieces of a page
template <int DH, int NT, int TYPE>
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(AttendArgs a, int blocks) {
    constexpr bool HALF = TYPE == ROWS_BF16;
    constexpr float BIAS = HALF ? 7.f : 0.f;
    constexpr int NQ = attend_nq<TYPE>, NP = attend_np<TYPE, HALF>, TD = DH / 64, DT = DH / 16;
    extern __shared__ u32x4 lds[];                               // [2] pages
    __shared__ int nan_seen[2][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % a.c.heads, rest = blockIdx.x / a.c.heads, b = rest % a.n_seqs, block = blocks - 1 - rest / a.n_seqs;
    const int group = a.n_heads / a.c.heads, r0 = block * 64 * NT;
    const AttendSeq s = uniform(attend_seq(a, b));
    const int R = s.rows * group, seen = s.seen;
    if (r0 >= R) return;
    const int r1 = r0 + 64 * NT < R ? r0 + 64 * NT : R, furthest = seen + (r1 - 1) / group;        // the block's last position
    const int pages = furthest < 0 ? 0 : furthest / PAGE_POS + 1;
    const int kb = lane >> 4, col = lane & 15, w0 = r0 + wave * 16 * NT;
    const int w1 = w0 + 16 * NT < R ? w0 + 16 * NT : R;
    const int wave_first = w0 < R ? seen + w0 / group : -1, wave_last = w0 < R ? seen + (w1 - 1) / group : -1, block_first = seen + r0 / group;
    const uint32_t k_off = (16 * (col >> 2) + (col & 3)) * DH + 16 * kb, v_off = col * PAGE_POS + 16 * kb;
    // ---- the wave's queries.  A negative scale turns their signs, so that the largest score is the largest product
    u32x4 q[NQ][NT][TD][2];
    const uint32_t turn = a.scale < 0.f ? 0x80008000u : 0u;
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = w0 + 16 * n + col;
        limit[n] = r < R ? seen + r / group : -1;
#pragma unroll
        for (int t = 0; t < TD; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
                for (int p = 0; p < NQ; ++p) q[p][n][t][h] = (u32x4){0, 0, 0, 0};
                if (r < R) {
                    const int row = s.row0 + r / group, hq = head * group + r % group, d = 64 * t + 16 * kb + 8 * h;
                    if constexpr (TYPE == ROWS_TILED) {
                        const size_t at = xtile_off(row, hq * DH + d, a.tile_ksp, a.quads);
                        q[0][n][t][h] = *(const u32x4 *)((const bf16_t *)a.q + at);
                        q[1][n][t][h] = *(const u32x4 *)((const bf16_t *)a.q_lo + at);
                    } else {
                        row8<TYPE>(a.q, (int64_t)row * a.q_row + hq * a.q_head + d, v);
#pragma unroll
                        for (int p = 0; p < NQ; ++p)
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                const uint32_t x = bf16_pair(v[2 * w], v[2 * w + 1]);
                                q[p][n][t][h][w] = x;
                                v[2 * w] -= __uint_as_float(x << 16);
                                v[2 * w + 1] -= __uint_as_float(x & 0xffff0000u);
                            }
                    }
#pragma unroll
                    for (int p = 0; p < NQ; ++p) q[p][n][t][h] ^= turn;
                }
            }
    }
    // ---- page numbers and scales, 64 pages a lane at a time: the present 64 and the next
    struct Pages { int id; float ks, vs; };
    const auto pages_from = [&](int i0) {
        Pages g{-1, 0.f, 0.f};
        const int i = i0 + lane;
        if (i < pages) g.id = a.table[(size_t)s.slot * a.max_blocks + i];
        if ((unsigned)g.id >= (unsigned)a.c.n_pages) g.id = -1;
        if (g.id >= 0) {
            g.ks = a.c.k_scale[(size_t)g.id * a.c.heads + head];
            g.vs = a.c.v_scale[(size_t)g.id * a.c.heads + head];
        }
        return g;
    };
    Pages now = pages_from(0), later = pages_from(64);
    int now_at = 0;                                              // the first page of `now`
    const auto id_of = [&](int i) { return i < now_at + 64 ? __builtin_amdgcn_readlane(now.id, i - now_at) : __builtin_amdgcn_readlane(later.id, i - now_at - 64); };
    const auto scale_of = [&](float x, float y, int i) {
        return __uint_as_float(i < now_at + 64 ? __builtin_amdgcn_readlane(__float_as_uint(x), i - now_at) : __builtin_amdgcn_readlane(__float_as_uint(y), i - now_at - 64));
    };
    // a thread's share of a page: score tile `wave`, feature tiles of V 4 u + wave
    u32x4 kc[TD], vc[DT / 4];
    const auto take = [&](int i) {
        const int id = id_of(i);
        const size_t at = ((size_t)(id < 0 ? 0 : id) * a.c.heads + head) * (PAGE_POS * DH);
#pragma unroll
        for (int t = 0; t < TD; ++t) kc[t] = *(const u32x4 *)((a.c.k + at + 4 * wave * DH + 64 * t) + k_off);
#pragma unroll
        for (int u = 0; u < DT / 4; ++u) vc[u] = *(const u32x4 *)((a.c.v + at + 16 * (4 * u + wave) * PAGE_POS) + v_off);
    };
    SumUnit unit{127, 67};                                       // of the page that was widened last
    const auto widen = [&](int i) {
        u32x4 *const to = lds + (i & 1) * rows_images<DH>;
#pragma unroll
        for (int t = 0; t < TD; ++t) {
            u32x4 lo, hi;
            widen16(kc[t], 1.f, lo, hi);
            to[((wave * TD + t) * 2) * 64 + lane] = lo;
            to[((wave * TD + t) * 2 + 1) * 64 + lane] = hi;
        }
        float vs = scale_of(now.vs, later.vs, i);
        if constexpr (HALF) vs = unit_factor(vs, unit);
        uint32_t nans = 0;
        if (i * PAGE_POS + PAGE_POS - 1 > block_first || id_of(i) < 0) {       // positions that some row does not see
            const int there = id_of(i) < 0 ? 0 : s.len - i * PAGE_POS - 16 * kb;
#pragma unroll
            for (int u = 0; u < DT / 4; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t c = vc[u][w] & bytes_below(there - 4 * w), m = nan_bytes(c);
                    nans |= m;
                    vc[u][w] = c & ~whole_bytes(m);
                }
        }
        nans = __ballot(nans != 0) != 0;
        if (lane == 0) nan_seen[i & 1][wave] = (int)nans;
#pragma unroll
        for (int u = 0; u < DT / 4; ++u) {
            u32x4 lo, hi;
            if constexpr (HALF) widen16_half(vc[u], vs, lo, hi);
            else widen16(vc[u], vs, lo, hi);
            to[4 * TD * 2 * 64 + ((4 * u + wave) * 2) * 64 + lane] = lo;
            to[4 * TD * 2 * 64 + ((4 * u + wave) * 2 + 1) * 64 + lane] = hi;
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
    const float to_log2 = fabsf(a.scale) * 1.44269504088896340736f;
    if (pages > 0) {
        take(0);
        widen(0);
        if (pages > 1) take(1);
    }
    __syncthreads();
    int o_unit = unit.now;                                       // that the wave's sums are in
    for (int i = 0; i < pages; ++i) {
        const int page_unit = unit.now;
        if (i + 1 < pages) widen(i + 1);
        if (i + 2 < pages) take(i + 2);
        const int base = i * PAGE_POS;
        if (base <= wave_last) {                                 // (the wave's rows see some of it)
            // operands come from LDS eight ahead of their products, V's first ones behind K's last
            constexpr int KI = 4 * TD * 2, VI = DT * 2;
            const u32x4 *const img = lds + (i & 1) * rows_images<DH> + lane;
            u32x4 w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = img[j * 64];
            const int id = id_of(i);
            const bool masked = id < 0 || base + PAGE_POS - 1 > wave_first;
            // (not 0: minus infinity has to stay that)
            const float by = fmaxf(to_log2 * scale_of(now.ks, later.ks, i), 1e-37f);
            u32x4 pb[NT][NP][2];
            f32x4 sc[NT][4];
            if (HALF && page_unit != o_unit) {                   // (exact)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] = times_pow2(o[n][d], o_unit - page_unit);
                o_unit = page_unit;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int g = 0; g < 4; ++g) sc[n][g] = (f32x4){0.f, 0.f, 0.f, 0.f};
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int j = 0; j < KI; ++j) {
                const int g = j / (2 * TD), t = j / 2 % TD, h = j % 2;
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p)
#pragma unroll
                    for (int n = 0; n < NT; ++n) sc[n][g] = mfma16x16x32(w[j % 8], q[p][n][t][h], sc[n][g]);
                w[j % 8] = img[(j + 8) * 64];
                __builtin_amdgcn_sched_group_barrier(0x008, NT * NQ, 0);       // (products, then a load: as written)
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_s_setprio(0);
            if (masked) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int left = (id < 0 ? -1 : limit[n]) - base - 16 * kb;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[n][e / 4][e % 4] = e > left ? LLMA_NEG_INF : sc[n][e / 4][e % 4];
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float top = LLMA_NEG_INF;
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[n][g][r]);
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
                        const int g = 2 * u + w / 2, r = 2 * (w & 1);
                        float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][g][r], by, -ref)), z = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][g][r + 1], by, -ref));
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            pb[n][p][u][w] = HALF ? half_pair(y, z) : bf16_pair(y, z);
                            if (p + 1 < NP) { y -= __uint_as_float(pb[n][p][u][w] << 16); z -= __uint_as_float(pb[n][p][u][w] & 0xffff0000u); }
                        }
                    }
            }
            // (taken out of the image where the block's first row does not see all of the page: also for waves whose rows all do)
            if (base + PAGE_POS - 1 > block_first && (nan_seen[i & 1][0] | nan_seen[i & 1][1] | nan_seen[i & 1][2] | nan_seen[i & 1][3]))
                attend_nans<DH, NT>(a.c.v + ((size_t)(id < 0 ? 0 : id) * a.c.heads + head) * (PAGE_POS * DH) + v_off, base, id < 0 ? 0 : s.len, limit, o);
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
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = w0 + 16 * n + col;
        if (r >= R) continue;
        const float inv = l[n][0] == 0.f ? 0.f : 1.f / l[n][0];
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const f32x4 v = o[n][d] * inv;
            attend_store<TYPE>(a, s.row0 + r / group, head * group + r % group, 16 * d + 4 * kb, HALF ? times_pow2(v, o_unit - 127) : v);
        }
    }
}

// a wave per row of a sequence that lies in several shares
template <int DH, int TYPE>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, AttendPlan plan) {
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

template <int DH, int NT, int TYPE>
static void launch_attend_nt(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
    const size_t bytes = (size_t)attend_lds<DH, NT, TYPE> + (size_t)(a.n_seqs + 1) * 4;
    hipLaunchKernelGGL((attend_paged_kernel<DH, NT, TYPE>), dim3((p.whole ? a.n_seqs : p.shares) * a.c.heads * p.tiles), dim3(256), bytes, st, a, p);
}
// row blocks of a call, at most: what blocks of 64 nt rows make of max_rows everywhere, or of all rows and a remainder per sequence
static int64_t attend_row_blocks(const AttendArgs &a, int nt) {
    const int64_t group = a.n_heads / a.c.heads, rows = 64 * nt;
    const int64_t by_max = a.n_seqs * ((a.max_rows * group + rows - 1) / rows), by_all = a.n_rows * group / rows + a.n_seqs;
    return (by_max < by_all ? by_max : by_all) * a.c.heads;
}
template <int DH, int NT, int TYPE>
static void launch_attend_rows(const AttendArgs &a, hipStream_t st) {
    const int group = a.n_heads / a.c.heads, blocks = (a.max_rows * group + 64 * NT - 1) / (64 * NT);
    hipLaunchKernelGGL((attend_rows_kernel<DH, NT, TYPE>), dim3((unsigned)blocks * a.n_seqs * a.c.heads), dim3(256), 2 * rows_images<DH> * 16, st, a, blocks);
}
template <int DH, int TYPE>
static void launch_attend_type(const AttendArgs &a, hipStream_t st) {
    constexpr int ROWS_NT = TYPE == ROWS_F32 ? 1 : 2;            // (three planes of queries and probabilities leave room for one tile)
    const int64_t group_rows = (int64_t)a.max_rows * (a.n_heads / a.c.heads), launched = (group_rows + 64 * ROWS_NT - 1) / (64 * ROWS_NT) * a.n_seqs * a.c.heads;
    if (group_rows > 64 && attend_row_blocks(a, ROWS_NT) >= ROWS_MIN && launched < 1 << 23) return launch_attend_rows<DH, ROWS_NT, TYPE>(a, st);
    const AttendPlan p = attend_plan(a.n_seqs, a.max_blocks, a.n_heads, a.c.heads, DH, a.max_rows);
    if (p.nt == 1) launch_attend_nt<DH, 1, TYPE>(a, p, st);
    else if (p.nt == 2) launch_attend_nt<DH, 2, TYPE>(a, p, st);
    else if (p.nt == 3) launch_attend_nt<DH, 3, TYPE>(a, p, st);
    else launch_attend_nt<DH, 4, TYPE>(a, p, st);
    if (p.shares > 1 && !p.whole)
        hipLaunchKernelGGL((attend_join_kernel<DH, TYPE>), dim3((a.max_rows * (a.n_heads / a.c.heads) + 3) / 4, a.c.heads, a.n_seqs), dim3(256), 0, st, a, p);
}
void launch_attend_paged(const AttendArgs &a, hipStream_t st) {
    if (a.n_seqs < 1 || a.n_rows < 1 || a.max_rows < 1) return;
    auto of = [&](auto dh) {
        constexpr int DH = decltype(dh)::value;
        if (a.type == ROWS_BF16) launch_attend_type<DH, ROWS_BF16>(a, st);
        else if (a.type == ROWS_F16) launch_attend_type<DH, ROWS_F16>(a, st);
        else if (a.type == ROWS_F32) launch_attend_type<DH, ROWS_F32>(a, st);
        else launch_attend_type<DH, ROWS_TILED>(a, st);
    };
    if (a.c.dh == 128) of(std::integral_constant<int, 128>{});
    else of(std::integral_constant<int, 64>{});
}
