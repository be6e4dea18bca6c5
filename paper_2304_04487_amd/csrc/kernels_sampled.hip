// Verification of drafted tokens against the target's probabilities, from given random numbers (speculative sampling).
//   p_j = softmax(logits_j / T), q_j the draft's distribution (one-hot where it is a copied token).  Draft j is accepted while u_j q_j(x_j) < p_j(x_j);
//   at the first rejection the token comes from max(p_j - q_j, 0), after all were accepted from p_k: the smallest v with
//   sum_{i <= v} w_i > r * sum w.  T <= 0: the arg max (lowest id), as the greedy step has it.
// Bound by one read of the logits.  That pass keeps maxima and fp32 sums of 2^x, which decide all but about one test in 10^4; a test too near its border
// for them is decided again with the row's sum in 64 bits.  The one row that is sampled is read again in 64 bits throughout, so that
// a token does not depend on how the sums were cut: exponentials off by 1e-7 would move one sample in some hundreds.
#include "../../include/llma.h"
#include "row_pieces.h"

#define ROW_THREADS 256
#define PICK_BLOCKS 512          // 16-byte pieces of a row per workgroup when it is sampled (two a thread)

__device__ __forceinline__ int drafts_of(const SampledArgs &a, int b) {
    const int n = a.n_draft ? a.n_draft[b] : a.k;
    return n < 0 ? 0 : n > a.k ? a.k : n;
}
__device__ __forceinline__ float temperature_of(const SampledArgs &a, int b) { return a.temperature ? a.temperature[b] : 1.f; }
// log2(e) / T, and twice that in fp32.  An infinite T takes all logits above minus infinity alike, the type's lowest among them, where a factor of 0 would make NaN of
// minus infinity, a masked logit, in place of no weight at all: its factors leave nothing of differences up to 2^129 (2^-71; in fp32 2^-21, which takes 4e-7 of a
// weight).
__device__ __forceinline__ double by64_of(float t) { return fmax(1.4426950408889634074 / (double)t, 0x1p-200); }
__device__ __forceinline__ float twice_by(float by) { return fmaxf(2.f * by, 0x1p-149f); }
// 2^((x - top) by), by halves: a difference of finite logits does not become infinite
__device__ __forceinline__ float part_of(float x, float top, float by2) { return __builtin_amdgcn_exp2f(__builtin_fmaf(0.5f, x, -0.5f * top) * by2); }
__device__ __forceinline__ float logit_of(float x) { return x != x ? LLMA_NEG_INF : x; }           // NaN: a token that cannot be
// A row's weights e^((x - top) / T) in 64 bits, as 2^((x - top) by), by = log2(e) / T.  2^f for |f| <= 1/2 by the polynomial of degree 10 that is 1 at 0 and meets it
// at the ten Chebyshev points of the interval (off by 6e-16 of it); a whole number is split off by adding 1.5 2^52, whose low word it becomes.
// The top itself counts 1, also an infinite one; minus infinity, NaN and what is below 2^-2000 count 0 (fmax passes over a NaN).
struct Weigher { float top; double by, least; };
__device__ __forceinline__ Weigher weigher(float top, double by) { return Weigher{top, by, -2000.0 / by}; }
__device__ __forceinline__ double weight64(float x, const Weigher &w) {
    constexpr double whole = 6755399441055744.0;
    const double d = fmax((double)x - (double)w.top, w.least);
    const double t = __builtin_fma(d, w.by, whole), f = __builtin_fma(d, w.by, whole - t);
    double p = 7.070977866508138e-09;
    p = __builtin_fma(p, f, 1.0205905413765595e-07);
    p = __builtin_fma(p, f, 1.3215451633221434e-06);
    p = __builtin_fma(p, f, 1.5252672924850737e-05);
    p = __builtin_fma(p, f, 0.00015403530424776529);
    p = __builtin_fma(p, f, 0.0013333558200794592);
    p = __builtin_fma(p, f, 0.009618129107618665);
    p = __builtin_fma(p, f, 0.05550410866465167);
    p = __builtin_fma(p, f, 0.24022650695910075);
    p = __builtin_fma(p, f, 0.6931471805599462);
    p = __builtin_fma(p, f, 1.0);
    p = __builtin_amdgcn_ldexp(p, (int)__double_as_longlong(t));
    return w.top == -LLMA_NEG_INF && x == w.top ? 1.0 : p;
}

struct RowPart { float top, sum; int where; };                   // of a chunk: maximum, sum of 2^((x - top) log2(e) / T), first index of the maximum

// work: RowPart[rows][chunks] | per sequence: Choice | double weight sums [n_seqs][picks] (and, with draft probabilities, exponentials' sums before them)
struct Choice { int accepted, row, token, residual; float top; int greedy; double sum, inv_sum; };

struct SampledPlan { int chunk_blocks, chunks, picks; int64_t at_choice, at_sums, bytes; };
static SampledPlan sampled_plan(int n_seqs, int k, int vocab, int epb) {
    SampledPlan p;
    const int64_t blocks = ((int64_t)vocab + epb - 1) / epb + 1, rows = (int64_t)n_seqs * (k + 1);       // (+ 1: a row that begins inside a piece)
    // eight pieces a thread where that leaves enough workgroups for the chip, two where it does not
    p.chunk_blocks = rows * ((blocks + 2047) / 2048) >= 1024 ? 2048 : 512;
    p.chunks = (int)((blocks + p.chunk_blocks - 1) / p.chunk_blocks);
    p.picks = (int)((blocks + PICK_BLOCKS - 1) / PICK_BLOCKS);
    p.at_choice = (rows * p.chunks * (int64_t)sizeof(RowPart) + 63) / 64 * 64;
    p.at_sums = p.at_choice + (n_seqs * (int64_t)sizeof(Choice) + 63) / 64 * 64;
    p.bytes = p.at_sums + 2 * (int64_t)n_seqs * p.picks * 8;
    return p;
}
int64_t verify_sampled_bytes(int n_seqs, int k, int vocab) {
    const SampledPlan a = sampled_plan(n_seqs, k, vocab, 4), b = sampled_plan(n_seqs, k, vocab, 8);
    return a.bytes > b.bytes ? a.bytes : b.bytes;
}

// A workgroup per chunk of a row: its maximum, then its sum, from registers.  Bound by the read: 64 sequences x 6 rows x 128256 bf16, 98 MB, 20.5 us = 4.8 TB/s;
// 16 x 33 x 32000 fp32, 68 MB, 14.3 us = 4.7; one sequence of 9 rows 3.4 us.
template <int NB, int TYPE>
__global__ __launch_bounds__(ROW_THREADS) void sampled_rows_kernel(SampledArgs a, SampledPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>;
    __shared__ RowPart parts[4];
    const int row = blockIdx.x, b = row / (a.k + 1), j = row % (a.k + 1), t = threadIdx.x, lane = t & 63;
    if (j > drafts_of(a, b)) return;                             // (a row that no draft leads to)
    const float temp = temperature_of(a, b);
    const bool greedy = !(temp > 0.f);
    const RowView v = row_view<TYPE>(a, row);
    const int blocks = (v.skip + a.vocab + EPB - 1) / EPB, first = blockIdx.y * plan.chunk_blocks;
    // the pieces stay as they come (unpacked twice they cost less than the registers of their values): requested together, then maximum, then sum
    u32x4 x[NB];
    float top = LLMA_NEG_INF;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int blk = first + i * ROW_THREADS + t;
        x[i] = v.base[blk < blocks ? blk : 0];
    }
    const int id0 = (first + t) * EPB - v.skip;                  // of the thread's first logit
    // all pieces of the chunk wholly the row's: nothing to mask
    const bool inside = first * EPB >= v.skip && (first + NB * ROW_THREADS) * (int64_t)EPB - v.skip <= a.vocab;
    const auto values = [&](int i, float (&f)[EPB]) {
        piece_values<TYPE>(x[i], f);
        if (!inside) {
#pragma unroll
            for (int e = 0; e < EPB; ++e) {
                const int id = id0 + i * ROW_THREADS * EPB + e;
                f[e] = id >= 0 && id < a.vocab ? f[e] : LLMA_NEG_INF;
            }
        }
    };
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        float f[EPB];
        values(i, f);
#pragma unroll
        for (int e = 0; e < EPB; ++e) top = fmaxf(top, f[e]);     // (passes over NaN)
    }
    butterfly<32>([&](auto o) { top = fmaxf(top, lane_xor<o.value>(top)); });
    if (lane == 0) parts[t >> 6].top = top;
    __syncthreads();
    top = fmaxf(fmaxf(parts[0].top, parts[1].top), fmaxf(parts[2].top, parts[3].top));
    // (or the compiler would keep the values of the first pass)
#pragma unroll
    for (int i = 0; i < NB; ++i) asm volatile("" : "+v"(x[i]));
    float sum = 0.f;
    int where = 0x7fffffff;
    if (greedy) {
#pragma unroll
        for (int i = NB - 1; i >= 0; --i) {
            float f[EPB];
            values(i, f);
#pragma unroll
            for (int e = EPB - 1; e >= 0; --e)
                if (f[e] == top && top != LLMA_NEG_INF) where = id0 + i * ROW_THREADS * EPB + e;
        }
        butterfly<32>([&](auto o) { const int w = lane_xor<o.value>(where); where = w < where ? w : where; });
    } else {
        const float by2 = twice_by(1.44269504088896340736f / temp);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            float f[EPB];
            values(i, f);
#pragma unroll
            for (int e = 0; e < EPB; ++e) sum += part_of(f[e], top, by2);
        }
        if (sum != sum) {                                        // a NaN among them, or an infinite top: token by token
            sum = 0.f;
#pragma unroll 1
            for (int i = 0; i < NB; ++i) {
                float f[EPB];
                const int blk = first + i * ROW_THREADS + t;
                piece_values<TYPE>(v.base[blk < blocks ? blk : 0], f);
#pragma unroll
                for (int e = 0; e < EPB; ++e) {
                    const int id = id0 + i * ROW_THREADS * EPB + e;
                    const float l = id >= 0 && id < a.vocab ? logit_of(f[e]) : LLMA_NEG_INF;
                    const float w = l == top ? 1.f : part_of(l, top, by2);
                    sum += l == LLMA_NEG_INF ? 0.f : w;
                }
            }
        }
        butterfly<32>([&](auto o) { sum += lane_xor<o.value>(sum); });
    }
    if (lane == 0) { parts[t >> 6].sum = sum; parts[t >> 6].where = where; }
    __syncthreads();
    if (t == 0) {
        RowPart p{top, 0.f, 0x7fffffff};
        for (int w = 0; w < 4; ++w) { p.sum += parts[w].sum; p.where = parts[w].where < p.where ? parts[w].where : p.where; }
        ((RowPart *)a.work)[(int64_t)row * plan.chunks + blockIdx.y] = p;
    }
}

template <int OFF> __device__ __forceinline__ double lane_xor64(double v) { return __longlong_as_double((long long)lane_xor<OFF>((unsigned long long)__double_as_longlong(v))); }
__device__ __forceinline__ double block_sum(double v, double *part) {       // over 256 threads; part: LDS of four words
    butterfly<32>([&](auto o) { v += lane_xor64<o.value>(v); });
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}
// inclusive prefix sum over 256 threads, *total the sum
__device__ __forceinline__ double scan64(double v, double *part, double *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double all = v;                              // of the lane's group of 1, 2, 4 .. lanes
    const auto step = [&](auto o) {
        const double other = lane_xor64<o.value>(all);
        if (lane & o.value) v += other;
        all += other;
    };
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 8>{});
    step(std::integral_constant<int, 16>{});
    step(std::integral_constant<int, 32>{});
    __syncthreads();
    if (lane == 0) part[wave] = all;
    __syncthreads();
    double before = 0.0, sum = 0.0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        before += w < wave ? part[w] : 0.0;
        sum += part[w];
    }
    *total = sum;
    return before + v;
}
template <int TYPE>
__device__ double row_sum64(const SampledArgs &a, int64_t row, float top, double by, double *part) {
    constexpr int EPB = sampled_epb<TYPE>;
    const RowView v = row_view<TYPE>(a, row);
    const int blocks = (v.skip + a.vocab + EPB - 1) / EPB;
    const Weigher weigh = weigher(top, by);
    double s = 0.0;
    for (int blk = threadIdx.x; blk < blocks; blk += 256) {
        float x[EPB];
        piece_values<TYPE>(v.base[blk], x);
#pragma unroll
        for (int e = 0; e < EPB; ++e) {
            const int id = blk * EPB - v.skip + e;
            if (id >= 0 && id < a.vocab) s += weight64(x[e], weigh);
        }
    }
    return block_sum(s, part);
}
template <int TYPE>
__device__ __forceinline__ float logit_at(const SampledArgs &a, int64_t row, int id) {
    const int64_t at = row * a.row_stride + id;
    if constexpr (TYPE == ROWS_F32) return logit_of(((const float *)a.logits)[at]);
    else if constexpr (TYPE == ROWS_F16) return logit_of((float)((const _Float16 *)a.logits)[at]);
    else return logit_of(bf16_to_f32(((const bf16_t *)a.logits)[at]));
}

// How many drafts of sequence b hold, and which row its token comes from.  All threads of a workgroup call it and get the same; lane j looks at row j.  The sums of the
// rows' chunks are fp32: a test whose sides are nearer than 3e-5 of each other, and 2^-24 for each chunk, is decided again with the row's sum in 64 bits.  (A chunk's
// sum is off by 5e-6 at most: 2e-7 of the exponent, which is up to 17 where weights still matter, 64 addends a thread, and its factor; each chunk that is added rounds
// the sum by half of 2^-23.  A row has up to 4096.)
template <int TYPE>
__device__ Choice decide(const SampledArgs &a, const SampledPlan &plan, int b, double *part) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)b * (a.k + 1) + lane;
    const bool in = lane <= a.k, tested = lane < a.k;
    // everything that needs no other value first: a row's chunks eight at a time (those of rows that no draft leads to hold anything)
    const RowPart *const p = (const RowPart *)a.work + (in ? row : (int64_t)b * (a.k + 1)) * plan.chunks;
    const float temp = temperature_of(a, b);
    int draft = -1;
    float q = 1.f, u = 0.f;
    if (tested) {
        draft = a.drafts[(int64_t)b * a.draft_stride + lane];
        u = a.u_accept[(int64_t)b * a.k + lane];
    }
    const int n_draft = drafts_of(a, b);
    const bool greedy = !(temp > 0.f);
    const double by64 = greedy ? 0.0 : by64_of(temp);
    const float by2 = twice_by((float)by64);
    const bool fits = tested && (unsigned)draft < (unsigned)a.vocab;
    const float logit = fits ? logit_at<TYPE>(a, row, draft) : 0.f;
    if (fits && a.probs) q = a.probs[((int64_t)b * a.k + lane) * a.vocab + draft];
    float top = LLMA_NEG_INF, sum = 0.f;
    int where = 0x7fffffff;
    for (int c0 = 0; c0 < plan.chunks; c0 += 8) {
        RowPart x[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = p[c0 + c < plan.chunks ? c0 + c : c0];
        float here = top;
#pragma unroll
        for (int c = 0; c < 8; ++c) here = fmaxf(here, x[c].top);
        // (a top that is infinite counts 1 by itself and leaves nothing to lower ones)
        sum *= top == here ? 1.f : part_of(top, here, by2);
        if (top != here) where = 0x7fffffff;
        if (top == LLMA_NEG_INF) sum = 0.f;
        top = here;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            if (c0 + c >= plan.chunks) continue;
            if (x[c].top == here && x[c].where < where) where = x[c].where;
            if (x[c].top > LLMA_NEG_INF) sum += x[c].sum * (x[c].top == here ? 1.f : part_of(x[c].top, here, by2));
        }
    }
    double left = 0.0, right = 0.0;                              // u q sum < e
    bool ok = false, near = false;
    if (lane < n_draft && fits && top > LLMA_NEG_INF) {
        if (greedy) {
            ok = draft == where;
        } else {
            right = weight64(logit, weigher(top, by64));
            left = (double)u * (double)q * (double)sum;
            ok = left < right;
            near = right > 0.0 && fabs(left - right) <= (3e-5 + plan.chunks * 0x1p-24) * right;
        }
    }
    unsigned long long yes = __ballot(ok), unsure = __ballot(near);
    // (the first rejection ends it: only tests before it matter)
    while (true) {
        const unsigned long long no = ~yes;
        const int stop = __builtin_ctzll(no);                    // lane n_draft <= 63 is never ok
        const unsigned long long look = unsure & ((2ull << stop) - 1);
        if (look == 0) break;
        const int j = __builtin_ctzll(look);
        unsure &= ~(1ull << j);
        const float tj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top), j));
        const double s = row_sum64<TYPE>(a, (int64_t)b * (a.k + 1) + j, tj, by64, part);
        const unsigned long long again = __ballot(lane == j && (double)u * (double)q * s < right);
        yes = (yes & ~(1ull << j)) | again;
    }
    const int n = __builtin_ctzll(~yes);
    Choice c;
    c.accepted = n;
    c.row = (int)((int64_t)b * (a.k + 1) + n);
    c.residual = n < n_draft;
    c.greedy = greedy;
    c.top = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top), n));
    c.token = c.residual ? __builtin_amdgcn_readlane(draft, n) : -1;       // the rejected draft
    if (greedy) c.token = __builtin_amdgcn_readlane(where, n);             // (0x7fffffff: nothing to choose)
    c.sum = c.inv_sum = 0.0;
    return c;
}

// the weights of a piece of the sampled row: e, or what is left of p once q is taken off
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
template <int TYPE>
__device__ __forceinline__ void piece_weights(const SampledArgs &a, const Choice &c, const RowView &v, int blocks, int blk, const Weigher &weigh, bool minus, const float *q, double w[sampled_epb<TYPE>]) {
    constexpr int EPB = sampled_epb<TYPE>;
    const int id0 = blk * EPB - v.skip;
    const bool edge = id0 < 0 || blk * (int64_t)EPB - v.skip + EPB > a.vocab;       // not wholly the row's
    float x[EPB], taken[EPB];
    piece_values<TYPE>(v.base[blk < blocks ? blk : 0], x);
    if (minus && q) {
        if (edge) {
#pragma unroll
            for (int e = 0; e < EPB; ++e) taken[e] = blk < blocks && id0 + e >= 0 && id0 + e < a.vocab ? q[id0 + e] : 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < EPB; e += 4) *(f32x4 *)(taken + e) = *(const f32x4_any *)(q + id0 + e);
        }
    }
    if (edge) {
#pragma unroll
        for (int e = 0; e < EPB; ++e) x[e] = blk < blocks && id0 + e >= 0 && id0 + e < a.vocab ? x[e] : LLMA_NEG_INF;
    }
#pragma unroll
    for (int e = 0; e < EPB; ++e) w[e] = weight64(x[e], weigh);
    if (minus) {
#pragma unroll
        for (int e = 0; e < EPB; ++e) w[e] = q ? fmax(__builtin_fma(w[e], c.inv_sum, -(double)taken[e]), 0.0) : id0 + e == c.token ? 0.0 : w[e];
    }
}

// a workgroup per (piece range of the sampled row, sequence): sums of its weights.  PASS 0 decides and sums the exponentials (without draft probabilities:
// the weights themselves); PASS 1, with draft probabilities, sums max(p - q, 0).
// Bound by the 64-bit instructions of the weights (18 each) and, where there are few, by the decision that every workgroup makes for itself: 64 sequences x 128256 15.2 us and,
// PASS 1, 13.5; one sequence x 32000 6.1.  Two ranges a workgroup: 2 % less at 64 sequences, 2 % more at 32.  The workgroup of a sequence's last sum going on to the token,
// in place of the next kernel: nothing for one sequence, twice the time for 64, whose workgroups all write back and invalidate their caches for it.
template <int TYPE, int PASS>
__global__ __launch_bounds__(256) void sampled_pick_kernel(SampledArgs a, SampledPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>;
    __shared__ double part[4];
    const int b = blockIdx.x;
    Choice *const choice = (Choice *)((char *)a.work + plan.at_choice) + b;
    double *const sums = (double *)((char *)a.work + plan.at_sums) + (int64_t)b * 2 * plan.picks;
    Choice c;
    if constexpr (PASS == 0) {
        c = decide<TYPE>(a, plan, b, part);
        if (blockIdx.y == 0 && threadIdx.x == 0) *choice = c;
    } else {
        c = *choice;
        if (!c.residual) return;
        double s = 0.0;
        for (int i = threadIdx.x; i < plan.picks; i += 256) s += sums[i];
        c.sum = block_sum(s, part);
        c.inv_sum = 1.0 / c.sum;
        if (blockIdx.y == 0 && threadIdx.x == 0) {                          // (the other fields are read by all, these by the next kernel)
            choice->sum = c.sum;
            choice->inv_sum = c.inv_sum;
        }
    }
    if (c.greedy) return;
    const Weigher weigh = weigher(c.top, by64_of(temperature_of(a, b)));
    const RowView v = row_view<TYPE>(a, c.row);
    const int blocks = (v.skip + a.vocab + EPB - 1) / EPB;
    const bool minus = PASS == 1 || (a.probs == nullptr && c.residual);
    const float *const q = PASS == 1 ? a.probs + ((int64_t)b * a.k + c.accepted) * a.vocab : nullptr;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < PICK_BLOCKS / 256; ++i) {
        double w[EPB];
        piece_weights<TYPE>(a, c, v, blocks, blockIdx.y * PICK_BLOCKS + i * 256 + threadIdx.x, weigh, minus, q, w);
#pragma unroll
        for (int e = 0; e < EPB; ++e) s += w[e];
    }
    s = block_sum(s, part);
    if (threadIdx.x == 0) sums[PASS * plan.picks + blockIdx.y] = s;
}

// The first thread, in order, whose `hit` is set hands its two values to the workgroup (2), else the last whose `some` is (1); 0 if there is neither.  slots: LDS of eight
struct Found { double at; int id; };
__device__ __forceinline__ int first_of(bool hit, bool some, double at, int id, Found *slots, Found *out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned long long hits = __ballot(hit), any = __ballot(some);
    const int who = hits ? __builtin_ctzll(hits) : any ? 63 - __builtin_clzll(any) : -1;
    if (lane == (who < 0 ? 0 : who)) slots[wave] = Found{at, who < 0 ? -1 : id};
    if (lane == 0) slots[4 + wave].id = hits != 0;
    __syncthreads();
    int best = -1;
#pragma unroll
    for (int w = 3; w >= 0; --w)
        if (slots[4 + w].id) best = w;
    const bool is_hit = best >= 0;
    if (!is_hit) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (slots[w].id >= 0) best = w;
    }
    if (best >= 0) *out = slots[best];
    return best < 0 ? 0 : is_hit ? 2 : 1;
}
// A workgroup per sequence: the range the random number falls into, then the token in it.  Bound by its chain: the choice and the ranges' sums, a scan, the range's
// pieces (8 or 16 exponentials a thread), a scan.  With separate sums and scans, and atomics that look for the first hit, one sequence over 32000 tokens took 9.8 us
// where it takes 4.1.
template <int TYPE>
__global__ __launch_bounds__(256) void sampled_finish_kernel(SampledArgs a, SampledPlan plan) {
    constexpr int EPB = sampled_epb<TYPE>, PER = PICK_BLOCKS / 256;
    __shared__ double part[4];
    __shared__ Found ranges[8], tokens[8];
    const int b = blockIdx.x, t = threadIdx.x;
    const double *const base = (const double *)((const char *)a.work + plan.at_sums) + (int64_t)b * 2 * plan.picks;
    // requested together: the choice, the first 256 ranges' sums of both passes, the random number, the drafts
    const Choice c = ((const Choice *)((const char *)a.work + plan.at_choice))[b];
    const double all0 = t < plan.picks ? base[t] : 0.0, left0 = a.probs && t < plan.picks ? base[plan.picks + t] : 0.0;
    const double u = (double)a.u_sample[b];
    const Weigher weigh = weigher(c.top, by64_of(temperature_of(a, b)));
    const int draft = t < a.k ? a.drafts[(int64_t)b * a.draft_stride + t] : -1;
    int token = -1;
    if (c.greedy) {
        token = c.token == 0x7fffffff ? -1 : c.token;
    } else {
        const bool with_q = c.residual && a.probs != nullptr;
        bool minus = c.residual, all = !with_q;                  // which weights, which sums
        const auto sum_of = [&](int i) { return i < plan.picks ? (i == t ? (all ? all0 : left0) : base[(all ? 0 : plan.picks) + i]) : 0.0; };
        double total, up_to, sum, first;                         // (up to 256 ranges: one scan gives both; first: the sum of the first 256)
        const auto add_up = [&]() {
            up_to = scan64(sum_of(t), part, &first);
            total = first;
            for (int i0 = 256; i0 < plan.picks; i0 += 256) total += block_sum(sum_of(i0 + t), part);
        };
        add_up();
        if (c.residual && !(total > 0.0)) {                      // p nowhere above q: p itself
            minus = false;
            if (with_q) {
                all = true;
                add_up();
            } else if (c.top > LLMA_NEG_INF) {
                token = c.token;                                 // (the rejected token is the only one there is)
            }
        }
        if (total > 0.0) {
            const double target = u * total;
            // the first range whose cumulative sum passes the target, else the last with a weight; what lies before it
            Found range{0.0, -1}, found{0.0, -1};
            double before = 0.0;
            for (int i0 = 0; i0 < plan.picks; i0 += 256) {
                const double w = sum_of(i0 + t);
                if (i0 > 0) {
                    __syncthreads();                             // (the last 256's answer has been read)
                    up_to = before + scan64(w, part, &sum);
                }
                const int is = first_of(w > 0.0 && up_to > target, w > 0.0, up_to - w, i0 + t, ranges, &found);
                if (is) range = found;
                if (is == 2) break;
                before += i0 == 0 ? first : sum;
            }
            const RowView v = row_view<TYPE>(a, c.row);
            const int blocks = (v.skip + a.vocab + EPB - 1) / EPB;
            const float *const q = with_q && minus ? a.probs + ((int64_t)b * a.k + c.accepted) * a.vocab : nullptr;
            // a thread's pieces are neighbours, so that cumulative sums run along the threads
            double w[PER][EPB], own = 0.0;
            const int blk0 = range.id * PICK_BLOCKS + t * PER;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                piece_weights<TYPE>(a, c, v, blocks, blk0 + i, weigh, minus, q, w[i]);
#pragma unroll
                for (int e = 0; e < EPB; ++e) own += w[i][e];
            }
            double run = range.at + scan64(own, part, &sum) - own;
            int mine = -1, last = -1;
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int e = 0; e < EPB; ++e) {
                    const int id = (blk0 + i) * EPB - v.skip + e;
                    run += w[i][e];
                    if (w[i][e] > 0.0) {
                        last = id;
                        if (run > target && mine < 0) mine = id;
                    }
                }
            if (first_of(mine >= 0, last >= 0, 0.0, mine >= 0 ? mine : last, tokens, &found)) token = found.id;
        }
    }
    if (t <= a.k) {
        int e = -1;
        if (t < c.accepted) e = draft;
        else if (t == c.accepted) e = token;
        a.emitted[(int64_t)b * a.emit_stride + t] = e;
    }
    if (t == 0) {
        a.n_accepted[b] = c.accepted;
        a.next[b] = token;
    }
}

template <int TYPE>
static void launch_sampled(const SampledArgs &a, hipStream_t st) {
    const SampledPlan p = sampled_plan(a.n_seqs, a.k, a.vocab, sampled_epb<TYPE>);
    const dim3 rows(a.n_seqs * (a.k + 1), p.chunks), picks(a.n_seqs, p.picks);
    if (p.chunk_blocks == 2048) hipLaunchKernelGGL((sampled_rows_kernel<8, TYPE>), rows, dim3(ROW_THREADS), 0, st, a, p);
    else hipLaunchKernelGGL((sampled_rows_kernel<2, TYPE>), rows, dim3(ROW_THREADS), 0, st, a, p);
    hipLaunchKernelGGL((sampled_pick_kernel<TYPE, 0>), picks, dim3(256), 0, st, a, p);
    if (a.probs) hipLaunchKernelGGL((sampled_pick_kernel<TYPE, 1>), picks, dim3(256), 0, st, a, p);
    hipLaunchKernelGGL((sampled_finish_kernel<TYPE>), dim3(a.n_seqs), dim3(256), 0, st, a, p);
}
void launch_verify_sampled(const SampledArgs &a, hipStream_t st) {
    if (a.type == ROWS_BF16) launch_sampled<ROWS_BF16>(a, st);
    else if (a.type == ROWS_F16) launch_sampled<ROWS_F16>(a, st);
    else launch_sampled<ROWS_F32>(a, st);
}

// ---------------------------------------------------------------------------------------------
// a context's sampled step
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void take_words_kernel(const int *pinned, int *dev, int words) {
    for (int i = threadIdx.x; i < words; i += 256) dev[i] = pinned[i];
}
void launch_take_words(const int *pinned, int *dev, int words, hipStream_t st) { hipLaunchKernelGGL(take_words_kernel, dim3(1), dim3(256), 0, st, pinned, dev, words); }

// The accepted rows stay in the cache (T += a + 1), the new token becomes the pending one.  A row without a token leaves its sequence as it was: the
// host sees the -1 and reports it.
__global__ __launch_bounds__(256) void commit_sampled_kernel(CommitArgs c) {
    for (int b = threadIdx.x; b < c.n_seqs; b += 256) {
        const int n = c.n_accepted[b], next = c.next[b], slot = c.batch_slots[b];
        for (int j = 0; j <= n; ++j)
            __hip_atomic_store(c.io_emit + (size_t)b * c.io_stride + j, c.emitted[(size_t)b * c.emit_stride + j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        __hip_atomic_store(c.io_nacc + b, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        __hip_atomic_store(c.io_next + b, next, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        if (next < 0) continue;
        c.T[slot] += n + 1;
        c.pending[slot] = next;
    }
}
void launch_commit_sampled(const CommitArgs &c, hipStream_t st) { hipLaunchKernelGGL(commit_sampled_kernel, dim3(1), dim3(256), 0, st, c); }
