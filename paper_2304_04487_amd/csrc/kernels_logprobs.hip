// Log probabilities of given tokens, with the distribution's entropy, the tokens' ranks and the likeliest alternatives.
//   p = softmax(x / T);  log p(t) = (x_t - M) / T - ln S,  H = ln S - (W / S) / T  with M = max x, S = sum e^((x - M) / T), W = sum e^((x - M) / T) (x - M);
//   rank = tokens before t in the order of falling logits, ties by rising id, whose first n_top are the alternatives.
// Bound by one read of the logits: workgroups take chunks of rows and leave (M, S, W, rank's count), in fp32, relative to the chunk's own maximum, and the maximum
// of every segment of 4 U pieces.  A second launch, a workgroup per row, joins them in 64 bits and in a fixed order.  The n_top-th largest segment maximum bounds the alternatives from
// below, so it reads again only segments that reach it: n_top of a few hundred.
#include "../../include/llma.h"
#include "row_pieces.h"

#define CHUNK_THREADS 256
#define TOP_KEPT 2048            // candidates that may wait; a batch adds up to 2048 more
#define TOP_LIST 1024            // segments that are looked through at a time

struct LogprobPlan { int u, chunks, segments; };                 // pieces a thread; chunks and segments of a row (64 a chunk)
static LogprobPlan logprob_plan(int n_rows, int vocab, int epb) {
    const int pieces = (vocab + epb - 1) / epb + 1;
    LogprobPlan p{8, 0, 0};
    const auto chunks = [&] { return (pieces + CHUNK_THREADS * p.u - 1) / (CHUNK_THREADS * p.u); };
    while (p.u > 1 && (int64_t)n_rows * chunks() < 1024) p.u /= 2;
    p.chunks = chunks();
    p.segments = 64 * p.chunks;
    return p;
}
static int64_t logprob_bytes(const LogprobPlan &p, int n_rows, int n_top) { return (int64_t)n_rows * (p.chunks * 16 + (n_top > 0 ? p.segments * 4 : 0)); }
int64_t token_logprobs_bytes(int n_rows, int vocab, int n_top) {
    const int64_t narrow = logprob_bytes(logprob_plan(n_rows, vocab, 8), n_rows, n_top), wide = logprob_bytes(logprob_plan(n_rows, vocab, 4), n_rows, n_top);
    return (narrow > wide ? narrow : wide) + 16;
}
struct LogprobPart { float m, s, w; int before; };

// e^((x - M) / T) as 2^((x - M) by), by = log2(e) / T in two parts: its own rounding would tilt all terms of a row alike
struct By { float hi, lo; double t; };
__device__ __forceinline__ By by_of(const LogprobArgs &a, int row) {
    float t = a.temperature ? a.temperature[row] : 1.f;
    if (!(t > 0.f)) t = 1.f;                                     // (also NaN)
    t = t > 3.402823466e38f ? 3.402823466e38f : t;
    const double by = 1.4426950408889634074 / (double)(t > 1e-37f ? t : 1e-37f);       // (below it only the maximum counts either way, and the range ends)
    By b;
    b.hi = (float)by;
    b.lo = (float)(by - (double)b.hi);
    b.t = (double)t;
    return b;
}
__device__ __forceinline__ float power(float d, const By &b) { return __builtin_amdgcn_exp2f(__builtin_fmaf(d, b.lo, d * b.hi)); }
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
// the smallest float above x (of plus infinity: NaN, which nothing reaches)
__device__ __forceinline__ float next_above(float x) {
    const int b = (int)__float_as_uint(x);
    if (x == -LLMA_NEG_INF) return __builtin_nanf("");
    if (x == 0.f) return __uint_as_float(1u);
    return __uint_as_float((uint32_t)(b < 0 ? b - 1 : b + 1));
}

template <int TYPE, int U>
__global__ __launch_bounds__(CHUNK_THREADS) void logprob_chunk_kernel(LogprobArgs a, LogprobPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>;
    __shared__ float tops[4];
    __shared__ LogprobPart parts[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x / plan.chunks, chunk = blockIdx.x % plan.chunks;
    const RowView view = row_view<TYPE>(a, row);
    const int pieces = (view.skip + a.vocab + EPB - 1) / EPB, p0 = chunk * CHUNK_THREADS * U + threadIdx.x;
    u32x4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = row_piece<TYPE>(view, p0 + u * CHUNK_THREADS, pieces, a.vocab);
    const By by = by_of(a, row);
    const int token = a.tokens ? a.tokens[row] : -1;
    const bool given = (unsigned)token < (unsigned)a.vocab;
    const float xt = given ? logit_at<TYPE>(a, row, token) : 0.f;
    // ---- maxima
    float top = LLMA_NEG_INF;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float x[EPB];
        piece_values<TYPE>(w[u], x);
#pragma unroll
        for (int e = 0; e < EPB; ++e) top = fmaxf(top, x[e]);    // (passes over NaN)
    }
    top = fmaxf(top, lane_xor<1>(top));
    top = fmaxf(top, lane_xor<2>(top));
    float *const segments = (float *)((LogprobPart *)a.work + (int64_t)a.n_rows * plan.chunks);
    if (a.n_top > 0 && lane % 4 == 0) segments[(int64_t)row * plan.segments + chunk * 64 + threadIdx.x / 4] = top;
    top = fmaxf(top, lane_xor<4>(top));
    butterfly<32>([&](auto o) { if constexpr (o.value >= 8) top = fmaxf(top, lane_xor<o.value>(top)); });
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    const float M = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    // ---- sums.  Tokens at or above the given one's logit count before it when their id is lower, tokens above it always
    const float above = given ? next_above(xt) : __builtin_nanf(""), same = given ? xt : __builtin_nanf("");
    const int pt = given ? (token + view.skip) / EPB : 0;
    // (far out: an infinite maximum, which counts 1 and all else 0, or a temperature whose inverse ends the range)
    const bool far = M == -LLMA_NEG_INF || by.hi < 1e-20f;
    float s = 0.f, sd = 0.f;
    int before = 0;
    if (far) {
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            float x[EPB];
            piece_values<TYPE>(row_piece<TYPE>(view, p0 + u * CHUNK_THREADS, pieces, a.vocab), x);
#pragma unroll
            for (int e = 0; e < EPB; ++e) {
                const float v = fmaxf(x[e], LLMA_NEG_INF), d = v == M ? 0.f : v - M, y = d == LLMA_NEG_INF ? 0.f : power(d, by);
                s += y;
                sd += y > 0.f ? y * d : 0.f;
            }
        }
    } else if (M != LLMA_NEG_INF) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[EPB];
            piece_values<TYPE>(w[u], x);
#pragma unroll
            for (int e = 0; e < EPB; ++e) {
                const float d = fmaxf(x[e] - M, -1e30f), y = power(d, by);       // (minus infinity and NaN: 0)
                s += y;
                sd = __builtin_fmaf(y, d, sd);
            }
        }
    }
    if (given && a.rank) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = p0 + u * CHUNK_THREADS;
            float x[EPB];
            piece_values<TYPE>(w[u], x);
            const float least = p < pt ? same : above;
            // (minus infinity, if that is what is given, counts too, and what is not the row's would)
            const int i0 = p * EPB - view.skip;
#pragma unroll
            for (int e = 0; e < EPB; ++e) {
                const float v = fmaxf(x[e], LLMA_NEG_INF);
                before += (v >= least || (p == pt && v == same && i0 + e < token)) && (same != LLMA_NEG_INF || (i0 + e >= 0 && i0 + e < a.vocab));
            }
        }
    }
    butterfly<32>([&](auto o) {
        s += lane_xor<o.value>(s);
        sd += lane_xor<o.value>(sd);
        before += lane_xor<o.value>(before);
    });
    if (lane == 0) parts[wave] = LogprobPart{0.f, s, sd, before};
    __syncthreads();
    if (threadIdx.x == 0) {
        LogprobPart t{M, 0.f, 0.f, 0};
        for (int i = 0; i < 4; ++i) {
            t.s += parts[i].s;
            t.w += parts[i].w;
            t.before += parts[i].before;
        }
        ((LogprobPart *)a.work)[(int64_t)row * plan.chunks + chunk] = t;
    }
}

// floats as integers of the same order; minus infinity is the least but one that can be, NaN is not asked
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);                 // (minus zero is zero)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// the n-th largest of `count` distinct keys in LDS, all threads of the workgroup
__device__ __forceinline__ unsigned long long nth_key(const unsigned long long *keys, int count, int n, int *sums) {
    unsigned long long t = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long c = t | 1ull << bit;
        int at = 0;
        for (int i = threadIdx.x; i < count; i += CHUNK_THREADS) at += keys[i] >= c;
        butterfly<32>([&](auto o) { at += lane_xor<o.value>(at); });
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = at;
        __syncthreads();
        if (sums[0] + sums[1] + sums[2] + sums[3] >= n) t = c;
    }
    return t;
}

template <int TYPE>
__global__ __launch_bounds__(CHUNK_THREADS) void logprob_row_kernel(LogprobArgs a, LogprobPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>;
    __shared__ float tops[4];
    __shared__ double sums[4][2];
    __shared__ int counts[4];
    __shared__ unsigned long long keys[TOP_KEPT + 8 * CHUNK_THREADS];
    __shared__ int list[TOP_LIST];
    __shared__ int n_keys, n_list, cut[4];
    __shared__ uint32_t least_segment;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x;
    const LogprobPart *const parts = (const LogprobPart *)a.work + (int64_t)row * plan.chunks;
    const By by = by_of(a, row);
    // ---- the chunks' sums, in 64 bits
    float top = LLMA_NEG_INF;
    for (int i = threadIdx.x; i < plan.chunks; i += CHUNK_THREADS) top = fmaxf(top, parts[i].m);
    butterfly<32>([&](auto o) { top = fmaxf(top, lane_xor<o.value>(top)); });
    if (lane == 0) tops[wave] = top;
    if (threadIdx.x == 0) n_keys = 0;
    __syncthreads();
    const float M = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    double s = 0., w = 0.;
    int before = 0;
    for (int i = threadIdx.x; i < plan.chunks; i += CHUNK_THREADS) {
        const LogprobPart p = parts[i];
        const float d = p.m == M ? 0.f : p.m - M, f = p.m == LLMA_NEG_INF || d == LLMA_NEG_INF ? 0.f : power(d, by);
        if (f > 0.f) {
            s += (double)f * p.s;
            w += (double)f * ((double)p.w + (double)d * p.s);
        }
        before += p.before;
    }
    butterfly<32>([&](auto o) {
        s += __longlong_as_double((long long)lane_xor<o.value>((unsigned long long)__double_as_longlong(s)));
        w += __longlong_as_double((long long)lane_xor<o.value>((unsigned long long)__double_as_longlong(w)));
        before += lane_xor<o.value>(before);
    });
    if (lane == 0) {
        sums[wave][0] = s;
        sums[wave][1] = w;
        counts[wave] = before;
    }
    __syncthreads();
    s = sums[0][0] + sums[1][0] + sums[2][0] + sums[3][0];
    const double log_s = s > 0. ? log(s) : 0.;
    const auto logprob_of = [&](float x) {
        if (x == LLMA_NEG_INF) return LLMA_NEG_INF;
        if (M == -LLMA_NEG_INF) return x == M ? (float)-log_s : LLMA_NEG_INF;
        return (float)(((double)x - (double)M) / by.t - log_s);
    };
    if (threadIdx.x == 0) {
        const int token = a.tokens ? a.tokens[row] : -1;
        const bool given = (unsigned)token < (unsigned)a.vocab;
        if (a.logprob) a.logprob[row] = given ? logprob_of(logit_at<TYPE>(a, row, token)) : LLMA_NEG_INF;
        if (a.rank) a.rank[row] = given ? counts[0] + counts[1] + counts[2] + counts[3] : -1;
        if (a.entropy) a.entropy[row] = s > 0. ? (float)(log_s - (sums[0][1] + sums[1][1] + sums[2][1] + sums[3][1]) / s / by.t) : 0.f;
    }
    if (a.n_top < 1) return;
    // ---- the n_top-th largest segment maximum: no alternative lies below it
    const float *const segments = (const float *)((const LogprobPart *)a.work + (int64_t)a.n_rows * plan.chunks) + (int64_t)row * plan.segments;
    if (wave == 0) {
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = t | 1u << bit;
            int n = 0;
            for (int i = lane; i < plan.segments; i += 64) n += ordered(segments[i]) >= c;
            butterfly<32>([&](auto o) { n += lane_xor<o.value>(n); });
            if (n >= a.n_top) t = c;
            if (n == a.n_top) break;
        }
        if (lane == 0) least_segment = t;
    }
    __syncthreads();
    const RowView view = row_view<TYPE>(a, row);
    const int pieces = (view.skip + a.vocab + EPB - 1) / EPB;
    const uint32_t nothing = ordered(LLMA_NEG_INF);
    const uint32_t reach = least_segment > nothing ? least_segment : nothing + 1;
    unsigned long long least = (unsigned long long)reach << 32;  // keys: the logit's order, then the lower id
    for (int g0 = 0; g0 < plan.segments; g0 += TOP_LIST) {
        __syncthreads();
        if (threadIdx.x == 0) n_list = 0;
        __syncthreads();
        for (int g = g0 + threadIdx.x; g < g0 + TOP_LIST && g < plan.segments; g += CHUNK_THREADS)
            if (ordered(segments[g]) >= reach) list[atomicAdd(&n_list, 1)] = g;
        __syncthreads();
        const int all = n_list * 4 * plan.u;
        for (int i0 = 0; i0 < all; i0 += CHUNK_THREADS) {
            const int i = i0 + threadIdx.x;
            if (i < all) {
                const int g = list[i / (4 * plan.u)], u = i / 4 % plan.u;
                const int p = (g / 64 * plan.u + u) * CHUNK_THREADS + g % 64 * 4 + i % 4;
                float x[EPB];
                piece_values<TYPE>(row_piece<TYPE>(view, p, pieces, a.vocab), x);
#pragma unroll
                for (int e = 0; e < EPB; ++e) {
                    const float v = fmaxf(x[e], LLMA_NEG_INF);
                    const unsigned long long key = (unsigned long long)ordered(v) << 32 | (0xffffffffu - (uint32_t)(p * EPB - view.skip + e));
                    if (key >= least) keys[atomicAdd(&n_keys, 1)] = key;
                }
            }
            __syncthreads();
            if (n_keys > TOP_KEPT) {                             // (many equal or rising logits) keep the n_top largest
                const int count = n_keys;
                least = nth_key(keys, count, a.n_top, cut);
                unsigned long long mine[(TOP_KEPT + 8 * CHUNK_THREADS) / CHUNK_THREADS];
#pragma unroll
                for (int k = 0; k < (TOP_KEPT + 8 * CHUNK_THREADS) / CHUNK_THREADS; ++k) mine[k] = k * CHUNK_THREADS + (int)threadIdx.x < count ? keys[k * CHUNK_THREADS + threadIdx.x] : 0;
                __syncthreads();
                if (threadIdx.x == 0) n_keys = 0;
                __syncthreads();
#pragma unroll
                for (int k = 0; k < (TOP_KEPT + 8 * CHUNK_THREADS) / CHUNK_THREADS; ++k)
                    if (mine[k] >= least) keys[atomicAdd(&n_keys, 1)] = mine[k];
                __syncthreads();
            }
            __syncthreads();
        }
    }
    __syncthreads();
    const int count = n_keys;
    if (count > 4 * LOGPROB_MAX_TOP) least = nth_key(keys, count, a.n_top, cut);
    int *const tokens = a.top_tokens + (int64_t)row * a.n_top;
    float *const logprobs = a.top_logprobs + (int64_t)row * a.n_top;
    for (int i = threadIdx.x; i < count; i += CHUNK_THREADS) {
        const unsigned long long key = keys[i];
        if (key < least) continue;
        int place = 0;
        for (int j = 0; j < count; ++j) place += keys[j] > key;
        if (place < a.n_top) {
            tokens[place] = (int)(0xffffffffu - (uint32_t)key);
            logprobs[place] = logprob_of(value_of((uint32_t)(key >> 32)));
        }
    }
    for (int i = count + threadIdx.x; i < a.n_top; i += CHUNK_THREADS) {
        tokens[i] = -1;
        logprobs[i] = LLMA_NEG_INF;
    }
}

void launch_token_logprobs(const LogprobArgs &a, hipStream_t st) {
    if (a.n_rows < 1) return;
    auto of = [&](auto type) {
        constexpr int TYPE = decltype(type)::value;
        const LogprobPlan p = logprob_plan(a.n_rows, a.vocab, sampled_epb<TYPE>);
        const dim3 grid((unsigned)((int64_t)a.n_rows * p.chunks)), block(CHUNK_THREADS);
        if (p.u == 8) hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 8>), grid, block, 0, st, a, p);
        else if (p.u == 4) hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 4>), grid, block, 0, st, a, p);
        else if (p.u == 2) hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 2>), grid, block, 0, st, a, p);
        else hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 1>), grid, block, 0, st, a, p);
        hipLaunchKernelGGL((logprob_row_kernel<TYPE>), dim3(a.n_rows), block, 0, st, a, p);
    };
    if (a.type == ROWS_BF16) of(std::integral_constant<int, ROWS_BF16>{});
    else if (a.type == ROWS_F16) of(std::integral_constant<int, ROWS_F16>{});
    else of(std::integral_constant<int, ROWS_F32>{});
}
