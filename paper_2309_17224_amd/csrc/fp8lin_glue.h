// Device helpers shared by the kernels of the decoder layer (fp8lin_decoder.hip)
// and of its key/value cache (fp8lin_cache.hip): bf16 words, the cast with a
// predicted bias, wave reductions and the bf16 matrix product.  Internal, not
// part of the ABI.
#pragma once

#include <type_traits>

#include "fp8lin_fp8.h"
#include "fp8lin_internal.h"

namespace fp8lin {
namespace {

constexpr int32_t kNoPrediction = INT32_MIN;  // never equal to a clamped bias

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint4 ld16(const void* p) { return *(const uint4*)p; }
__device__ __forceinline__ void st16(void* p, uint4 v) { *(uint4*)p = v; }

// Eight bf16 values (four packed words) -> eight codes with bias b; NaN
// inputs are re-encoded as the casts do.
template <int FMT>
__device__ __forceinline__ uint2 codes8(uint4 v, int b) {
    uint32_t lo = cast4_bf16<FMT>(v.x, v.y, b), hi = cast4_bf16<FMT>(v.z, v.w, b);
    if (__builtin_expect(any_nan_bf16(v.x, v.y) || any_nan_bf16(v.z, v.w), 0)) {
        const uint32_t h0[4] = {v.x & 0xFFFFu, v.x >> 16, v.y & 0xFFFFu, v.y >> 16};
        const uint32_t h1[4] = {v.z & 0xFFFFu, v.z >> 16, v.w & 0xFFFFu, v.w >> 16};
        lo = nan_patch<FMT>(lo, h0);
        hi = nan_patch<FMT>(hi, h1);
    }
    return make_uint2(lo, hi);
}

// Largest magnitude pattern of eight bf16 values.
__device__ __forceinline__ uint32_t mag8(uint4 v) {
    us2 m = {0, 0};
    m = fold_bf16(m, v);
    return max((uint32_t)m.x, (uint32_t)m.y);
}

// The bias the fused cast uses: the prediction, clamped as the casts clamp.
// Block 0 records it for the check kernel (kNoPrediction without one, which
// makes the check kernel cast every element).
__device__ __forceinline__ int fused_bias(const int32_t* pred, int32_t* used) {
    const int b = pred ? clamp_bias(*pred) : 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *used = pred ? b : kNoPrediction;
    return b;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

__device__ __forceinline__ f4_t mfma_bf16(u32x4 a, u32x4 b, f4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                   c, 0, 0, 0);
}

__device__ __forceinline__ u32x4 ldg16(const uint16_t* p) { return *(const u32x4*)p; }

// 32-bit LDS address of a pointer into a __shared__ array.
__device__ __forceinline__ uint32_t lds_addr32(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// Maximum / sum over lanes l, l ^ 16, l ^ 32, l ^ 48 (the four lanes that hold
// one query's scores) with VALU lane swaps: swapping a value with itself
// between rows 0-1 and 2-3 of 16 lanes (then between the two halves of the
// wave) leaves each lane holding its own value and its partner's, in some
// order, which a symmetric operation does not see.
__device__ __forceinline__ float quad_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int V> using IC = std::integral_constant<int, V>;

template <typename Fn>
void with_fmt(int fmt, Fn&& fn) {
    switch (fmt) {
        case FP8_E4M3: fn(IC<FP8_E4M3>{}); break;
        case FP8_E5M2: fn(IC<FP8_E5M2>{}); break;
        case FP8_E4_A: fn(IC<FP8_E4_A>{}); break;
        default: fn(IC<FP8_E5_A>{}); break;
    }
}

}  // namespace
}  // namespace fp8lin
