// Log probabilities of given tokens, with the distribution's entropy, the tokens' ranks and the likeliest alternatives.
//   p = softmax(x / T);  log p(t) = (x_t - M) / T - ln S,  H = ln S - (W / S) / T  with M = max x, S = sum e^((x - M) / T), W = sum e^((x - M) / T) (x - M);
//   rank = tokens before t in the order of falling logits, ties by rising id, whose first n_top are the alternatives.
// Bound by one read of the logits: each wave takes a chunk of a row, all of it in registers, and leaves (R, S, W, the rank's count): sums of 2^t and 2^t t with t = x
// by - R, by = log2(e) / T, R near the chunk's largest x by; and the maximum of every segment (16 or more pieces that lie together).  A second launch, a wave per row,
// joins them in 64 bits and in a fixed order.  The n_top-th largest segment maximum bounds the alternatives from below, so it reads again only segments that reach it.
// 2000 rows of 128256 bf16, 513 MB, 20 alternatives: 103 us = 5.0 TB/s and 23 us; the same reads alone take 82, the rest of the first launch is eleven vector
// instructions a logit.  Its second half (row by row) is the chain of bound, segments and places, and 6 KB of scattered reads a row.  Nine rows of 32000 fp32, 5
// alternatives: 3.6 and 9.8 us, of which an empty launch is 2 and half the fetching of code.
#include "../../include/llma.h"
#include "row_pieces.h"

#define CHUNK_PIECES(u) (64 * (u))                               // of a wave
#define TOP_KEPT 256             // candidates that may wait; a piece a lane adds up to 512
#define TOP_FEW 24               // alternatives
#define TOP_AHEAD 4              // pieces a lane requests at once when it looks for them
#define TOP_LIST 1024            // segments whose maxima a wave keeps in registers, and looks through at a time
#define LOW (-1e30f)             // logits are raised to this where only sums and maxima are meant: its products stay finite where minus infinity would end sums in NaN, and NaN goes with it

struct LogprobPlan { int u, lanes, chunks, segments; };          // pieces a lane; lanes of a segment; chunks and segments of a row
static LogprobPlan logprob_plan(int n_rows, int vocab, int epb) {
    const int pieces = (vocab + epb - 1) / epb + 1;
    LogprobPlan p{4, 16, 0, 0};                                  // (2000 rows of 128256 bf16, both launches: eight 127 us, four 122, two 148)
    const auto chunks = [&] { return (pieces + CHUNK_PIECES(p.u) - 1) / CHUNK_PIECES(p.u); };
    while (p.u > 1 && (int64_t)n_rows * chunks() < 4096) p.u /= 2;
    p.chunks = chunks();
    while (p.lanes < 64 && p.chunks * p.u * (64 / p.lanes) > TOP_LIST) p.lanes *= 2;
    p.segments = p.chunks * p.u * (64 / p.lanes);
    return p;
}
struct LogprobPart { double r; float s, w, hi; int before, pad[2]; };        // hi: what stood for by in fp32 (0: the sums were taken with by itself)
static int64_t logprob_bytes(const LogprobPlan &p, int n_rows, int n_top) { return (int64_t)n_rows * (p.chunks * (int64_t)sizeof(LogprobPart) + (n_top > 0 ? p.segments * 4ll : 0)); }
int64_t token_logprobs_bytes(int n_rows, int vocab, int n_top) {
    const int64_t narrow = logprob_bytes(logprob_plan(n_rows, vocab, 8), n_rows, n_top), wide = logprob_bytes(logprob_plan(n_rows, vocab, 4), n_rows, n_top);
    return (narrow > wide ? narrow : wide) + 16;
}

// T as it counts (infinite: all tokens with a logit above minus infinity alike), and by = log2(e) / T in 64 bits.  The chunks' sums are taken with an fp32 number near
// by, whose error tilts all terms of a row alike and is put right when the parts are joined
__device__ __forceinline__ float temperature_of(const LogprobArgs &a, int row) {
    const float t = a.temperature ? a.temperature[row] : 1.f;
    return t > 0.f ? t : 1.f;                                    // (NaN too)
}
__device__ __forceinline__ double by_of(float t) { return 1.4426950408889634074 / (double)t; }
template <int TYPE> __device__ __forceinline__ float logit_at(const LogprobArgs &a, int64_t row, int i) {
    const int64_t at = row * a.row_stride + i;
    float x;
    if constexpr (TYPE == ROWS_F32) x = ((const float *)a.logits)[at];
    else if constexpr (TYPE == ROWS_F16) x = (float)((const _Float16 *)a.logits)[at];
    else x = bf16_to_f32(((const bf16_t *)a.logits)[at]);
    return fmaxf(x, LLMA_NEG_INF);                               // NaN: a token that cannot be
}
// piece p of a row, minus infinity where it is not the row's
template <int TYPE>
__device__ __forceinline__ u32x4 row_piece(const RowView &v, int p, int pieces, int vocab) {
    constexpr int EPB = sampled_epb<TYPE>;
    constexpr uint32_t NONE = TYPE == ROWS_F32 ? 0xff800000u : TYPE == ROWS_F16 ? 0xfc00fc00u : 0xff80ff80u;
    u32x4 w = (u32x4){NONE, NONE, NONE, NONE};
    if (p < pieces) w = v.base[p];
    const int i0 = p * EPB - v.skip;
    if (p < pieces && (i0 < 0 || i0 + EPB > vocab)) {
#pragma unroll
        for (int e = 0; e < EPB; ++e)
            if (i0 + e < 0 || i0 + e >= vocab) {
                if constexpr (TYPE == ROWS_F32) w[e] = NONE;
                else w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | (NONE & 0xffff0000u) : (w[e / 2] & 0xffff0000u) | (NONE & 0xffffu);
            }
    }
    return w;
}
// x by, rounded: where logits are so large that this rounding shows, R has it too.  (by is 0 at an infinite temperature, where an infinite x stays that)
__device__ __forceinline__ double times_by(double x, double by) {
#pragma clang fp contract(off)
    const double z = x * by;
    return fabs(x) < __builtin_huge_val() ? z : x;
}
// the smallest float above x (of plus infinity: NaN, which nothing reaches)
__device__ __forceinline__ float next_above(float x) {
    const int b = (int)__float_as_uint(x);
    if (x == -LLMA_NEG_INF) return __builtin_nanf("");
    if (x == 0.f) return __uint_as_float(1u);
    return __uint_as_float((uint32_t)(b < 0 ? b - 1 : b + 1));
}
// of numbers that are no NaN (fmaxf would first quiet both)
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
// N numbers a lane of which each 16 lanes want the maxima: halves of the numbers go to halves of the lanes; lane l of 16 ends with number l N / 16
template <int N, int BIT = 8>
__device__ __forceinline__ float maxima16(const float (&m)[N]) {
    float h[N > 1 ? N / 2 : 1];
    if constexpr (N > 1) {
        const bool upper = threadIdx.x & BIT;
#pragma unroll
        for (int u = 0; u < N / 2; ++u) h[u] = larger(upper ? m[u + N / 2] : m[u], lane_xor<BIT>(upper ? m[u] : m[u + N / 2]));
    } else h[0] = larger(m[0], lane_xor<BIT>(m[0]));
    if constexpr (BIT > 1) return maxima16<(N > 1 ? N / 2 : 1), BIT / 2>(h);
    else return h[0];
}
// Over the wave, op of its two halves being the same either way: four steps inside 16 lanes (moves that the operation takes along), then 16 and 32 lanes swapped for a
// copy's.  (Steps by lane_xor need three instructions more to pick each lane's of the two, and a maximum of floats quiets both arguments first: a third of what a wave
// spends besides its logits)
template <typename F>
__device__ __forceinline__ int over_wave(int v, F op) {
    v = op(v, __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true));         // (eight lanes on)
    v = op(v, __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true));         // (eight lanes mirrored)
    v = op(v, __builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true));          // (two lanes on, of four; one)
    v = op(v, __builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true));
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return op((int)b[0], (int)b[1]);
}
__device__ __forceinline__ float sum_of_wave(float x) {
    return __int_as_float(over_wave(__float_as_int(x), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
// (of numbers that are no NaN, in the order of integers; the same in all lanes)
__device__ __forceinline__ float max_of_wave(float x) {
    int k = __float_as_int(x);
    k = over_wave(k ^ (k >> 31 & 0x7fffffff), [](int a, int b) { return a > b ? a : b; });
    k = __builtin_amdgcn_readfirstlane(k);
    return __int_as_float(k ^ (k >> 31 & 0x7fffffff));
}
template <typename F>
__device__ __forceinline__ void add_over_wave(F &v) {
    butterfly<32>([&](auto o) {
        if constexpr (std::is_same_v<F, double>) v += __longlong_as_double((long long)lane_xor<o.value>((unsigned long long)__double_as_longlong(v)));
        else v += lane_xor<o.value>(v);
    });
}

// a maximum with any NaN, also a signalling one, is the other number from here on
__device__ __forceinline__ void ieee_mode_off() { __builtin_amdgcn_s_setreg(1 | 9 << 6, 0); }      // (bit 9 of the mode register)

template <int TYPE, int U>
__global__ __launch_bounds__(256) void logprob_chunk_kernel(LogprobArgs a, LogprobPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>, N = U * EPB;
    ieee_mode_off();
    const int lane = threadIdx.x & 63;
    // (32 bits: a call's rows have at most 2^40 logits and a chunk of many rows 2^10.  A 64-bit division would be a sixth of a wave's instructions)
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= (uint32_t)a.n_rows * (uint32_t)plan.chunks) return;
    const int row = (int)(id / (uint32_t)plan.chunks), chunk = (int)(id % (uint32_t)plan.chunks);
    const RowView view = row_view<TYPE>(a, row);
    const int pieces = (view.skip + a.vocab + EPB - 1) / EPB, p0 = chunk * CHUNK_PIECES(U);
    u32x4 w[U];
    // (only a row's first and last chunk hold what is not the row's)
    if (p0 * EPB >= view.skip && (p0 + CHUNK_PIECES(U)) * EPB - view.skip <= a.vocab) {
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = view.base[p0 + 64 * u + lane];
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = row_piece<TYPE>(view, p0 + 64 * u + lane, pieces, a.vocab);
    }
    // (hi: any number near by will do, the part names it; one step of Newton's takes it to a rounding.  Where that leaves fp32, or T is infinite, it is no number or 0,
    // and the sums are taken with by itself)
    const float T = temperature_of(a, row), near = __builtin_amdgcn_rcpf(T), about = 1.4426950408889634f * near, hi = __builtin_fmaf(__builtin_fmaf(-T, about, 1.4426950408889634f), near, about);
    const int token = a.tokens ? a.tokens[row] : -1;
    const bool given = a.rank && (unsigned)token < (unsigned)a.vocab;
    const float xt = given ? logit_at<TYPE>(a, row, token) : 0.f;
    float x[N], m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        piece_values<TYPE>(w[u], x + u * EPB);
        m[u] = LOW;
#pragma unroll
        for (int e = 0; e < EPB; ++e) {
            asm("v_max_f32 %0, %1, %2" : "=v"(x[u * EPB + e]) : "v"(x[u * EPB + e]), "s"(LOW));       // (as fmaxf, which would first quiet its argument; one that is NaN gives way either way)
            m[u] = fmaxf(m[u], x[u * EPB + e]);
        }
    }
    // ---- maxima of segments, of the chunk
    float M = m[0];
#pragma unroll
    for (int u = 1; u < U; ++u) M = fmaxf(M, m[u]);
    float lowest = m[0];
#pragma unroll
    for (int u = 1; u < U; ++u) lowest = fminf(lowest, m[u]);
    if (__ballot(lowest <= LOW) != 0) {                          // (a piece all masked: by minus infinity, or by something between)
        M = LLMA_NEG_INF;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[EPB];                                        // (read again: kept, the pieces would cost the registers of a wave in four)
            piece_values<TYPE>(row_piece<TYPE>(view, p0 + 64 * u + lane, pieces, a.vocab), v);
            m[u] = LLMA_NEG_INF;
#pragma unroll
            for (int e = 0; e < EPB; ++e) m[u] = fmaxf(m[u], v[e]);
            M = fmaxf(M, m[u]);
        }
    }
    if (a.n_top > 0) {
        const int log_lanes = __builtin_ctz(plan.lanes);
        float *const segments = (float *)((LogprobPart *)a.work + (int64_t)a.n_rows * plan.chunks) + (int64_t)row * plan.segments + (chunk * U << (6 - log_lanes));
        float mine = maxima16<U>(m);
        if (plan.lanes >= 32) mine = fmaxf(mine, lane_xor<16>(mine));
        if (plan.lanes >= 64) mine = fmaxf(mine, lane_xor<32>(mine));
        if ((lane & (16 / U - 1)) == 0 && (lane & (plan.lanes - 1)) < 16) segments[((lane & 15) / (16 / U) << (6 - log_lanes)) + (lane >> log_lanes)] = mine;
    }
    M = max_of_wave(M);
    // ---- sums
    double R = LLMA_NEG_INF;
    float s = 0.f, sw = 0.f, taken = 0.f;
    const float r = M * hi;
    // (hi has an upper end too: LOW times it has to stay finite, or 0 times minus infinity would make the second sum NaN)
    if (fabsf(M) < 1e30f && hi > 1e-20f && hi < 1e8f && fabsf(r) < 4096.f) {
        R = (double)r;
        taken = hi;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float t = __builtin_fmaf(x[i], hi, -r), y = __builtin_amdgcn_exp2f(t);
            s += y;
            sw = __builtin_fmaf(y, t, sw);
        }
    } else if (M != LLMA_NEG_INF) {                              // an infinite maximum (it counts 1, all else 0), large logits, cold or very hot rows: in 64 bits up to 2^t
        const double by = by_of(T);
        R = times_by(M, by);
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            float v[EPB];
            piece_values<TYPE>(row_piece<TYPE>(view, p0 + 64 * u + lane, pieces, a.vocab), v);
#pragma unroll
            for (int e = 0; e < EPB; ++e) {
                const float z = fmaxf(v[e], LLMA_NEG_INF);
                const double t = z == M ? 0. : times_by((double)z - (double)M, by);
                const float y = t < -1000. ? 0.f : __builtin_amdgcn_exp2f((float)t);
                s += y;
                sw += y > 0.f ? y * (float)t : 0.f;
            }
        }
    }
    // ---- tokens before the given one: those above it, and as large ones with a lower id
    int before = 0;
    if (given) {
        const float above = next_above(xt);
        const int pt = (token + view.skip) / EPB;
        if (xt > LOW) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = p0 + 64 * u;
                if (pt >= p && pt < p + 64) {                    // (of the wave's pieces here)
#pragma unroll
                    for (int e = 0; e < EPB; ++e) {
                        const float v = x[u * EPB + e];
                        before += __popcll(__ballot(v >= above || (v == xt && (p + lane) * EPB + e < token + view.skip)));
                    }
                } else {
                    const float least = p > pt ? above : xt;
                    if (__ballot(m[u] >= least) == 0) continue;  // (m: of lanes, or of their 16: few reach a token that is likely)
#pragma unroll
                    for (int e = 0; e < EPB; ++e) before += __popcll(__ballot(x[u * EPB + e] >= least));
                }
            }
        } else {
#pragma unroll 1
            for (int u = 0; u < U; ++u) {
                const int i0 = (p0 + 64 * u + lane) * EPB - view.skip;
                float v[EPB];
                piece_values<TYPE>(row_piece<TYPE>(view, p0 + 64 * u + lane, pieces, a.vocab), v);
#pragma unroll
                for (int e = 0; e < EPB; ++e) {
                    const float z = fmaxf(v[e], LLMA_NEG_INF);
                    before += __popcll(__ballot((z >= above || (z == xt && i0 + e < token)) && i0 + e >= 0 && i0 + e < a.vocab));
                }
            }
        }
    }
    s = sum_of_wave(s);
    sw = sum_of_wave(sw);
    if (lane == 0) {
        LogprobPart t;
        t.r = R;
        t.s = s;
        t.w = sw;
        t.hi = taken;
        t.before = before;
        t.pad[0] = t.pad[1] = 0;
        ((LogprobPart *)a.work)[id] = t;
    }
}

// floats as integers of the same order
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);                 // (minus zero is zero)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// the n-th largest of `count` distinct keys in LDS
__device__ __forceinline__ unsigned long long nth_key(const unsigned long long *keys, int count, int n) {
    unsigned long long t = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long c = t | 1ull << bit;
        int at = 0;
        for (int i = 0; i < count; i += 64) {
            const int j = i + (int)threadIdx.x;
            at += __popcll(__ballot(j < count && keys[j < count ? j : 0] >= c));
        }
        if (at >= n) t = c;
    }
    return t;
}

template <int TYPE>
__global__ __launch_bounds__(64) void logprob_row_kernel(LogprobArgs a, LogprobPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>, HELD = TOP_LIST / 64;
    __shared__ unsigned long long keys[TOP_KEPT + 64 * EPB];
    __shared__ int list[TOP_LIST];
    __shared__ u32x4 ahead[TOP_AHEAD][64];
    __shared__ int ahead_at[TOP_AHEAD][64];
    ieee_mode_off();
    const int lane = threadIdx.x, row = blockIdx.x;
    const LogprobPart *const parts = (const LogprobPart *)a.work + (int64_t)row * plan.chunks;
    const float *const segments = (const float *)((const LogprobPart *)a.work + (int64_t)a.n_rows * plan.chunks) + (int64_t)row * plan.segments;
    uint32_t held[HELD];                                         // the first TOP_LIST segments' maxima; 0 for none, below all that can be
    if (a.n_top > 0) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) held[k] = k * 64 + lane < plan.segments ? ordered(segments[k * 64 + lane]) : 0u;
    }
    const double by = by_of(temperature_of(a, row));
    const int token = a.tokens ? a.tokens[row] : -1;
    const bool given = (unsigned)token < (unsigned)a.vocab;
    const float xt = given ? logit_at<TYPE>(a, row, token) : LLMA_NEG_INF;
    // ---- the chunks' sums, in 64 bits, relative to the largest R
    double R = LLMA_NEG_INF, s = 0., w = 0.;
    int before = 0;
    for (int i = lane; i < plan.chunks; i += 64) R = fmax(R, parts[i].r);
    butterfly<32>([&](auto o) { R = fmax(R, __longlong_as_double((long long)lane_xor<o.value>((unsigned long long)__double_as_longlong(R)))); });
    for (int i = lane; i < plan.chunks; i += 64) {
        const LogprobPart p = parts[i];
        const double d = p.r == R ? 0. : p.r - R;
        if (d > -1000.) {
            // A term is 2^(x hi) for 2^(x by): S lacks ln2 (by - hi) sum 2^t x, W that times the mean of t, and the sum itself (the spread of t, of the
            // size of (by - hi) too, is left out: 2^-24 of it; |x hi| is below 2^12, so the squares are 2^-24 at most, at logits of thousands).
            // (Exponential and logarithm in fp32, of numbers near 1: off by 2^-23 of a part, which 64 bits would not notice in the result)
            const double f = (double)__builtin_amdgcn_exp2f((float)d);
            const double lack = p.hi != 0.f ? (by / (double)p.hi - 1.) * (p.w + p.r * p.s) : 0., mean = p.hi != 0.f ? (double)(p.w / p.s) : 0.;
            const double ps = p.s + 0.69314718055994530942 * lack, pw = p.w + lack * (1. + 0.69314718055994530942 * mean);
            s += f * ps;
            w += f * (pw + d * ps);
        }
        before += p.before;
    }
    add_over_wave(s);
    add_over_wave(w);
    add_over_wave(before);
    const double log2_s = s > 0. ? (double)__builtin_amdgcn_logf((float)__builtin_amdgcn_frexp_mant(s)) + (double)__builtin_amdgcn_frexp_exp(s) : 0., ln2 = 0.69314718055994530942;
    const bool infinite = R == -(double)LLMA_NEG_INF;
    const auto minus_r = [&](double z) {
#pragma clang fp contract(off)
        return z - R;
    };
    const auto logprob_of = [&](float v) {
        if (v == LLMA_NEG_INF || (infinite && v != -LLMA_NEG_INF)) return LLMA_NEG_INF;
        return (float)(ln2 * ((infinite ? 0. : minus_r(times_by(v, by))) - log2_s));
    };
    if (lane == 0) {
        if (a.logprob) a.logprob[row] = logprob_of(xt);
        if (a.rank) a.rank[row] = given ? before : -1;
        if (a.entropy) a.entropy[row] = s > 0. ? (float)(ln2 * (log2_s - w / s)) : 0.f;
    }
    if (a.n_top < 1) return;
    // ---- a bound that at least n_top segments' maxima reach, few more: no alternative lies below it.  Of few alternatives the lanes' own maxima will do: an eighth of the
    // comparisons, and a fifth more segments that reach the bound (20 alternatives of 1002 segments: 24)
    uint32_t reach = 0;
    {
        const bool few = a.n_top <= TOP_FEW;
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < HELD; ++k) most = held[k] > most ? held[k] : most;
        if (plan.segments > TOP_LIST)
            for (int i = TOP_LIST + lane; i < plan.segments; i += 64) {
                const uint32_t c = ordered(segments[i]);
                most = c > most ? c : most;
            }
        uint32_t above = most;                                   // (bits above the highest that the lanes' maxima do not share need no test)
        if (few) {
            uint32_t low = most;
            butterfly<32>([&](auto o) {
                const uint32_t m = (uint32_t)lane_xor<o.value>((int)above), l = (uint32_t)lane_xor<o.value>((int)low);
                above = m > above ? m : above;
                low = l < low ? l : low;
            });
            above ^= low;
            reach = low;
        } else above = ~0u;
        const int bits = above == 0 ? 0 : 32 - __builtin_clz(above);
        reach = bits == 32 ? 0u : reach >> bits << bits;
        for (int bit = bits - 1; bit >= 0; --bit) {
            const uint32_t c = reach | 1u << bit;
            int n = 0;
            if (few) n = __popcll(__ballot(most >= c));
            else if (plan.segments <= TOP_LIST) {
#pragma unroll
                for (int k = 0; k < HELD; ++k) n += __popcll(__ballot(held[k] >= c));
            } else {
                for (int i = 0; i < plan.segments; i += 64) n += __popcll(__ballot(i + lane < plan.segments && ordered(segments[i + lane < plan.segments ? i + lane : 0]) >= c));
            }
            if (n >= a.n_top) reach = c;
            if (n >= a.n_top && n <= a.n_top + (few ? 0 : 4)) break;
        }
    }
    const RowView view = row_view<TYPE>(a, row);
    const int pieces = (view.skip + a.vocab + EPB - 1) / EPB;
    const uint32_t nothing = ordered(LLMA_NEG_INF);
    reach = reach > nothing ? reach : nothing + 1;
    unsigned long long least = (unsigned long long)reach << 32;  // keys: the logit's order, then the lower id
    const int log_each = __builtin_ctz(plan.lanes);              // a segment's pieces, a power of two; segments lie as pieces do
    int n_keys = 0;
    for (int g0 = 0; g0 < plan.segments; g0 += TOP_LIST) {
        // the segments that reach it, in order
        int n_list = 0;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int g = g0 + 64 * k + lane;
            const bool in = g < plan.segments && (g0 == 0 ? held[k] : ordered(segments[g < plan.segments ? g : 0])) >= reach;
            const unsigned long long all = __ballot(in);
            if (in) list[n_list + __popcll(all & ((1ull << lane) - 1))] = g;
            n_list += __popcll(all);
        }
        __syncthreads();
        const int n_pieces = n_list << log_each;
        for (int i0 = 0; i0 < n_pieces; i0 += TOP_AHEAD * 64) {
            // (through LDS, for short code: a call of a few rows spends its time on fetching it)
            u32x4 piece[TOP_AHEAD];
            int at[TOP_AHEAD];
#pragma unroll
            for (int k = 0; k < TOP_AHEAD; ++k) {
                const int i = i0 + 64 * k + lane, g = list[i < n_pieces ? i >> log_each : 0];
                at[k] = (g << log_each) + (i & (plan.lanes - 1));
                at[k] = i < n_pieces && at[k] < pieces ? at[k] : -1;
                piece[k] = view.base[at[k] < 0 ? 0 : at[k]];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < TOP_AHEAD; ++k) {
                ahead[k][lane] = piece[k];
                ahead_at[k][lane] = at[k];
            }
#pragma unroll 1
            for (int k = 0; k < TOP_AHEAD && i0 + 64 * k < n_pieces; ++k) {
                const float floor = value_of((uint32_t)(least >> 32));
                const int first = ahead_at[k][lane] * EPB - view.skip;
                float x[EPB], top = LLMA_NEG_INF;
                piece_values<TYPE>(ahead[k][lane], x);
#pragma unroll
                for (int e = 0; e < EPB; ++e) top = fmaxf(top, x[e]);
                if (ahead_at[k][lane] < 0) top = LLMA_NEG_INF;
                if (__ballot(top >= floor) == 0) continue;
                // (a row's first and last piece hold what is not the row's)
                uint32_t in = 0;
#pragma unroll
                for (int e = 0; e < EPB; ++e) in |= (top >= floor && x[e] >= floor && (unsigned)(first + e) < (unsigned)a.vocab ? 1u : 0u) << e;
                while (__ballot(in != 0) != 0) {                 // (one a lane at a time: hardly any lane has two)
                    const int e = in ? __builtin_ctz(in) : 0;
                    float v;
                    if constexpr (TYPE == ROWS_F32) v = ((const float *)&ahead[k][lane])[e];
                    else if constexpr (TYPE == ROWS_F16) v = (float)((const _Float16 *)&ahead[k][lane])[e];
                    else v = bf16_to_f32(((const bf16_t *)&ahead[k][lane])[e]);
                    const unsigned long long key = (unsigned long long)ordered(v) << 32 | (0xffffffffu - (uint32_t)(first + e));
                    const bool put = in != 0 && key >= least;
                    const unsigned long long all = __ballot(put);
                    if (put) keys[n_keys + __popcll(all & ((1ull << lane) - 1))] = key;
                    n_keys += __popcll(all);
                    in &= in - 1;
                }
                if (n_keys > TOP_KEPT) {                         // (many equal or rising logits) keep the n_top largest
                    __syncthreads();
                    least = nth_key(keys, n_keys, a.n_top);
                    int n = 0;
                    for (int i = 0; i < n_keys; i += 64) {       // (each round writes where it or one before it has read)
                        const unsigned long long key = i + lane < n_keys ? keys[i + lane] : 0;
                        const unsigned long long all = __ballot(key >= least);
                        __syncthreads();
                        if (key >= least) keys[n + __popcll(all & ((1ull << lane) - 1))] = key;
                        __syncthreads();
                        n += __popcll(all);
                    }
                    n_keys = n;
                }
            }
        }
        __syncthreads();
    }
    const int count = n_keys;
    if (count > 4 * LOGPROB_MAX_TOP) least = nth_key(keys, count, a.n_top);
    int *const tokens = a.top_tokens + (int64_t)row * a.n_top;
    float *const logprobs = a.top_logprobs + (int64_t)row * a.n_top;
    for (int i = lane; i < count; i += 64) {
        const unsigned long long key = keys[i];
        if (key < least) continue;
        int place = 0;
#pragma unroll 4
        for (int j = 0; j < count; ++j) place += keys[j] > key;
        if (place < a.n_top) {
            tokens[place] = (int)(0xffffffffu - (uint32_t)key);
            logprobs[place] = logprob_of(value_of((uint32_t)(key >> 32)));
        }
    }
    for (int i = count + lane; i < a.n_top; i += 64) {
        tokens[i] = -1;
        logprobs[i] = LLMA_NEG_INF;
    }
}

void launch_token_logprobs(const LogprobArgs &a, hipStream_t st) {
    if (a.n_rows < 1) return;
    auto of = [&](auto type) {
        constexpr int TYPE = decltype(type)::value;
        const LogprobPlan p = logprob_plan(a.n_rows, a.vocab, sampled_epb<TYPE>);
        const dim3 grid((unsigned)(((int64_t)a.n_rows * p.chunks + 3) / 4)), block(256);
        if (p.u == 4) hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 4>), grid, block, 0, st, a, p);
        else if (p.u == 2) hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 2>), grid, block, 0, st, a, p);
        else hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 1>), grid, block, 0, st, a, p);
        hipLaunchKernelGGL((logprob_row_kernel<TYPE>), dim3(a.n_rows), dim3(64), 0, st, a, p);
    };
    if (a.type == ROWS_BF16) of(std::integral_constant<int, ROWS_BF16>{});
    else if (a.type == ROWS_F16) of(std::integral_constant<int, ROWS_F16>{});
    else of(std::integral_constant<int, ROWS_F32>{});
}
