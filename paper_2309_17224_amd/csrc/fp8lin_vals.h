// Vectors of consecutive bf16 or fp32 values at any alignment, with a tail.
// Internal, not part of the ABI.
#pragma once

#include "fp8lin_fp8.h"

namespace fp8lin {
namespace {

// W consecutive values at p (any alignment), the first nv of them valid; the
// rest read as 0.
template <int W>
__device__ __forceinline__ void ld_bf16(const uint16_t* p, int nv, float (&v)[W]) {
    if (nv >= W) {
        uint32_t w[W / 2];
        if (W == 8) {
            const uint4 x = ld16_any(p);
            w[0] = x.x, w[1] = x.y, w[W / 2 - 2] = x.z, w[W / 2 - 1] = x.w;
        } else {
            const u32x2_any x = *(const u32x2_any*)p;
            w[0] = x.x, w[1] = x.y;
        }
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < nv ? __uint_as_float((uint32_t)p[i] << 16) : 0.0f;
    }
}

template <int W>
__device__ __forceinline__ void ld_vals(const void* base, int64_t at, int dt, int nv, float (&v)[W]) {
    if (dt == FP8_DT_BF16) {
        ld_bf16<W>((const uint16_t*)base + at, nv, v);
        return;
    }
    const float* p = (const float*)base + at;
    if (nv >= W) {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const uint4 x = ld16_any(p + i);
            v[i] = __uint_as_float(x.x), v[i + 1] = __uint_as_float(x.y);
            v[i + 2] = __uint_as_float(x.z), v[i + 3] = __uint_as_float(x.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < nv ? p[i] : 0.0f;
    }
}

template <int W>
__device__ __forceinline__ void st_bf16(uint16_t* p, int nv, const float (&v)[W]) {
    uint32_t w[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    if (nv >= W) {
        if (W == 8) st_stream(p, make_uint4(w[0], w[1], w[W / 2 - 2], w[W / 2 - 1]));
        else st8_any(p, w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < nv) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

template <int W>
__device__ __forceinline__ void st_vals(void* base, int64_t at, int dt, int nv, const float (&v)[W]) {
    if (dt == FP8_DT_BF16) {
        st_bf16<W>((uint16_t*)base + at, nv, v);
        return;
    }
    float* p = (float*)base + at;
    if (nv >= W) {
#pragma unroll
        for (int i = 0; i < W; i += 4)
            st_stream(p + i, make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]),
                                        __float_as_uint(v[i + 3])));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < nv) p[i] = v[i];
    }
}

// Four words of four codes, one a row -> four words, one a column.
__device__ __forceinline__ void transpose4(uint32_t (&r)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
    r[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    r[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    r[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    r[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

}  // namespace
}  // namespace fp8lin
