// Activations and the epilogues of the feed-forward matmuls (fp8lin_ffn.hip,
// fp8lin_ffn_small.hip): what happens to one row's consecutive columns once
// their sums are complete.  Internal, not part of the ABI.
#pragma once

#include "fp8lin_mm.h"
#include "fp8lin_vals.h"

namespace fp8lin {
namespace {

constexpr bool epi_fwd(int mode) { return mode == kEpiAct || mode == kEpiGlu; }
constexpr int epi_fa(int mode) { return epi_fwd(mode) ? FP8_E4M3 : FP8_E5M2; }  // format of A (B: E4M3)

// The VALU is what bounds the epilogues that have an exponential (a workgroup's 256
// x 256 outputs: about 0.4 us an operation of each, 1.6 us an exponential or
// reciprocal), so the forms below are the shortest that keep infinities, NaN and, relative
// to the value (of a slope, to its two terms), an error of (1 + |p| / 4) 2^-20 where the
// exponential is 2^-p: its argument's rounding, the larger the further out.  Exponentials
// and reciprocals below 2^-126 are 0: then |x| 2^-125 of a value is lost, and of a slope as
// much of either term.  act(-inf) = 0, act(inf) = inf, slopes 0 and 1.
constexpr float kMaxF = 3.402823466e38f;

// h = Phi(-a) = (1 - erf(a / sqrt 2)) / 2, a = |x|: e = exp(-a^2 / 2) times half the
// scaled complementary error function of a / sqrt 2, which is within 2.5e-7 of P(s),
// s = 1 / (1 + 0.255 a), for a <= 13.2, where e ends (the smallest largest relative error,
// by a linear program over 3000 points; 6e-7 in fp32), so the tail keeps its relative
// accuracy.  e is left in *e, P in *p.
__device__ __forceinline__ void gauss_tail(float x, float* e, float* p) {
    *e = __builtin_amdgcn_exp2f(x * -0.72134752f * x);
    const float s = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.255f, 1.0f));
    float q = fmaf(-0.0861081492f, s, 0.300115732f);
    q = fmaf(q, s, -0.213540407f);
    q = fmaf(q, s, 0.251808977f);
    q = fmaf(q, s, 0.0317131988f);
    q = fmaf(q, s, 0.115948818f);
    q = fmaf(q, s, 0.0999695562f);
    *p = fmaf(q, s, 9.23959189e-05f);
}

// q = 2^-p and sigma(p ln 2) = 1 / (1 + q).
__device__ __forceinline__ float sigma2(float p, float* q) {
    *q = __builtin_amdgcn_exp2f(-p);
    return __builtin_amdgcn_rcpf(1.0f + *q);
}

// f = act(x), d = act'(x) (what is not used costs nothing).
// GELU: x Phi(x) = max(x, 0) - a h; its slope Phi(x) + x phi(x) is k = e (P - a /
// sqrt(2 pi)) for x < 0 and 1 - k otherwise.
// The others are x sigma(p(x)), with slope sigma (1 + x p' (1 - sigma)), 1 - sigma = q sigma
// (with an infinite q sigma is 0, and q only has to be finite).
template <int ACT>
__device__ __forceinline__ void act_t(float x, float* f, float* d) {
    if constexpr (ACT == FP8_ACT_GELU) {
        float e, p;
        gauss_tail(x, &e, &p);
        *f = fmaf(-fminf(fabsf(x), kMaxF), p * e, fmaxf(x, 0.0f));
        const float k = e * fmaf(fminf(fabsf(x), 100.0f), -0.39894228f, p);
        *d = x < 0.0f ? k : 1.0f - k;
    } else if constexpr (ACT == FP8_ACT_GELU_TANH) {  // (1 + tanh u) / 2 = sigma(2 u), u = sqrt(2/pi) (x + 0.044715 x^3)
        float q;
        const float r = sigma2(x * fmaf(x * x, 0.1029432397f, 2.302208198f), &q);  // 2 sqrt(2/pi) log2(e) {0.044715, 1}
        *f = fmaxf(x, -kMaxF) * r;
        const float c = __builtin_amdgcn_fmed3f(x, -100.0f, 100.0f);
        const float dp = c * fmaf(c * c, 0.2140644488f, 1.595769122f);  // 2 sqrt(2/pi) {3 * 0.044715, 1}
        *d = fmaf(dp, fminf(q, kMaxF) * r, 1.0f) * r;
    } else if constexpr (ACT == FP8_ACT_SILU) {
        float q;
        const float r = sigma2(x * 1.442695041f, &q);
        *f = fmaxf(x, -kMaxF) * r;
        *d = fmaf(__builtin_amdgcn_fmed3f(x, -1000.0f, 1000.0f), fminf(q, kMaxF) * r, 1.0f) * r;
    } else if constexpr (ACT == FP8_ACT_RELU) {
        *f = x <= 0.0f ? 0.0f : x;
        *d = x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;
    } else {
        *f = x;
        *d = 1.0f;
    }
}

__device__ __forceinline__ void act_of(int act, float x, float* f, float* d) {
    switch (act) {
        case FP8_ACT_GELU: act_t<FP8_ACT_GELU>(x, f, d); break;
        case FP8_ACT_GELU_TANH: act_t<FP8_ACT_GELU_TANH>(x, f, d); break;
        case FP8_ACT_SILU: act_t<FP8_ACT_SILU>(x, f, d); break;
        case FP8_ACT_RELU: act_t<FP8_ACT_RELU>(x, f, d); break;
        default: act_t<FP8_ACT_NONE>(x, f, d);
    }
}

// Columns n .. n + W - 1 (nv of them valid) of row m: t the unscaled sums (with
// kEpiGlu the gate's, u the up projection's).  Every output is rounded once,
// from fp32.  The column sums of a backward epilogue are added to sa (with
// kEpiGluBwd: the gate's, sb the up projection's).  y: the output before its rounding
// (with kEpiGluBwd the gate's, x the up projection's).
template <int MODE, int W>
__device__ __forceinline__ void epi_row(const Epi& e, int64_t m, int64_t n, int nv, float (&t)[W], float (&u)[W],
                                        float (&sa)[W], float (&sb)[W], float (&y)[W], float (&x)[W]) {
    float f, d;
    if (epi_fwd(MODE)) {
        if (e.bias) {
            ld_vals<W>(e.bias, n, e.bias_dt, nv, x);
#pragma unroll
            for (int i = 0; i < W; ++i) t[i] += x[i];
            if (MODE == kEpiGlu) {
                ld_vals<W>(e.bias, e.N + n, e.bias_dt, nv, x);
#pragma unroll
                for (int i = 0; i < W; ++i) u[i] += x[i];
            }
        }
        if (e.keep) {
            st_bf16<W>(e.keep + m * e.ldkeep + n, nv, t);
            if (MODE == kEpiGlu) st_bf16<W>(e.keep + m * e.ldkeep + e.N + n, nv, u);
        }
        if (MODE == kEpiAct && e.res) ld_vals<W>(e.res, m * e.ldres + n, e.out_dt, nv, x);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            act_of(e.act, t[i], &f, &d);
            y[i] = MODE == kEpiGlu ? f * u[i] : e.res ? f + x[i] : f;
        }
        st_vals<W>(e.out, m * e.ldo + n, e.out_dt, nv, y);
    } else if (MODE == kEpiActBwd) {
        ld_bf16<W>(e.z + m * e.ldz + n, nv, x);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            act_of(e.act, x[i], &f, &d);
            y[i] = t[i] * d;
            sa[i] += y[i];
        }
        st_bf16<W>((uint16_t*)e.out + m * e.ldo + n, nv, y);
    } else {
        ld_bf16<W>(e.z + m * e.ldz + n, nv, x);
        ld_bf16<W>(e.z + m * e.ldz + e.N + n, nv, u);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            act_of(e.act, x[i], &f, &d);
            y[i] = t[i] * u[i] * d;
            x[i] = t[i] * f;
            sa[i] += y[i];
            sb[i] += x[i];
        }
        st_bf16<W>((uint16_t*)e.out + m * e.ldo + n, nv, y);
        st_bf16<W>((uint16_t*)e.out + m * e.ldo + e.N + n, nv, x);
    }
}

}  // namespace
}  // namespace fp8lin
