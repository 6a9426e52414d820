// Sums of rows of partial column sums, in an order that the number of rows alone sets.
// Internal, not part of the ABI.
#pragma once

#include "fp8lin_fp8.h"

namespace fp8lin {
namespace {

// out[col] = sum of the rows of part [rows, cols] for columns c0 .. c0 + 63, of type dt
// (columns from n0 on go to out1; either may be null): sixteen sums, of every 16th row
// each, eight loads under way, over the WAVES waves of the block; then those in order.
template <int WAVES>
__device__ __forceinline__ void sum_rows64(float (&red)[16][64], const float* __restrict__ part, int rows, int64_t cols,
                                           int64_t c0, void* out0, int64_t n0, void* out1, int dt) {
    const int c = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = c0 + c;
    const float* p = part + min(col, cols - 1);
#pragma unroll
    for (int s = w; s < 16; s += WAVES) {
        float v = 0.0f;
        for (int r0 = s; r0 < rows; r0 += 128) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = p[(int64_t)min(r0 + 16 * k, rows - 1) * cols];
#pragma unroll
            for (int k = 0; k < 8; ++k) v += r0 + 16 * k < rows ? x[k] : 0.0f;
        }
        red[s][c] = v;
    }
    __syncthreads();
    void* out = col < n0 ? out0 : out1;
    if (w == 0 && col < cols && out) {
        float v = red[0][c];
#pragma unroll
        for (int k = 1; k < 16; ++k) v += red[k][c];
        const int64_t at = col < n0 ? col : col - n0;
        if (dt == FP8_DT_BF16) ((uint16_t*)out)[at] = (uint16_t)(pack_bf16x2(v, 0.0f) & 0xFFFFu);
        else ((float*)out)[at] = v;
    }
    __syncthreads();  // red may be written again
}

}  // namespace
}  // namespace fp8lin
