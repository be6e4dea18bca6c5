// Rows of logits as their kernels read them (kernels_sampled.hip, kernels_logprobs.hip).
#pragma once
#include "paged.h"

template <int TYPE> constexpr int sampled_epb = TYPE == ROWS_F32 ? 4 : 8;        // logits of a 16-byte piece

// Rows begin anywhere: a row is read in the aligned 16-byte pieces that hold it, and what of the first and last is not its own is masked
// (both pieces hold a byte of the row, so they lie in its allocation).
struct RowView { const u32x4 *base; int skip; };                // pieces from the one with the row's first logit; logits before it in there
template <int TYPE, typename A>
__device__ __forceinline__ RowView row_view(const A &a, int64_t row) {
    constexpr int SIZE = TYPE == ROWS_F32 ? 4 : 2;
    // (from the pointer, not from an integer: loads through that would be flat ones)
    const char *const at = (const char *)a.logits + row * a.row_stride * SIZE;
    const int skip = (int)((uintptr_t)at & 15);
    return RowView{(const u32x4 *)(at - skip), skip / SIZE};
}
template <int TYPE>
__device__ __forceinline__ void piece_values(u32x4 p, float v[sampled_epb<TYPE>]) {
    if constexpr (TYPE == ROWS_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(p[e]);
    } else if constexpr (TYPE == ROWS_F16) {
        typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
        const f16x8 h = __builtin_bit_cast(f16x8, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(p[e] << 16); v[2 * e + 1] = __uint_as_float(p[e] & 0xffff0000u); }
    }
}
