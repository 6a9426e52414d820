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

// Phi(x) = (1 + erf(x / sqrt 2)) / 2 = 1 - Phi(-x): for a = |x| it is h = e^(-a^2/2)
// times half the scaled complementary error function of a / sqrt 2, which is
// within 4e-9 of s P(s), s = 1 / (1 + 0.24 a), for a <= 20 (a least-squares fit,
// reweighted towards the smallest largest relative error; 5e-7 in fp32), so the
// tail keeps its relative accuracy.
__device__ __forceinline__ float half_erfcx(float a) {
    const float s = __builtin_amdgcn_rcpf(1.0f + 0.24f * a);
    float p = 2.548838668e-02f;
    p = fmaf(p, s, -1.244845439e-01f);
    p = fmaf(p, s, 2.052491748e-01f);
    p = fmaf(p, s, -1.441438550e-01f);
    p = fmaf(p, s, 1.415055771e-01f);
    p = fmaf(p, s, 2.803383015e-02f);
    p = fmaf(p, s, 8.783841470e-02f);
    p = fmaf(p, s, 8.890991091e-02f);
    p = fmaf(p, s, 9.586130313e-02f);
    p = fmaf(p, s, 9.574180156e-02f);
    return p * s;
}

// x within [-top, top]; NaN stays.
__device__ __forceinline__ float within(float x, float top) { return x < -top ? -top : x > top ? top : x; }

// sigma(p ln 2) and sigma (1 - sigma), both to a few ulp at either end.
__device__ __forceinline__ void sigmoid2(float p, float* s, float* ds) {
    const float q = __builtin_amdgcn_exp2f(-fabsf(p)), r = __builtin_amdgcn_rcpf(1.0f + q);
    *s = p < 0.0f ? q * r : r;
    *ds = q * r * r;
}

// f = act(x), d = act'(x).  Beyond the clamps the exponentials are 0 in fp32;
// they keep infinities (act(-inf) = -0, act(inf) = inf, slopes 0 and 1).
__device__ __forceinline__ void act_of(int act, float x, float* f, float* d) {
    if (act == FP8_ACT_GELU) {
        const float c = within(x, 20.0f), e = __builtin_amdgcn_exp2f(c * c * -0.72134752f);
        const float h = half_erfcx(fabsf(c)) * e, phi = c < 0.0f ? h : 1.0f - h;
        *f = (x < 0.0f ? c : x) * phi;
        *d = fmaf(c * e, 0.39894228f, phi);
    } else if (act == FP8_ACT_GELU_TANH) {  // (1 + tanh u) / 2 = sigma(2 u), u = sqrt(2/pi) (x + 0.044715 x^3)
        const float c = within(x, 20.0f), c2 = c * c;
        float s, ds;
        sigmoid2(c * fmaf(c2, 0.1029432397f, 2.302208198f), &s, &ds);  // 2 sqrt(2/pi) log2(e) {0.044715, 1}
        *f = (x < 0.0f ? c : x) * s;
        *d = fmaf(c * ds, fmaf(c2, 0.2140644488f, 1.595769122f), s);   // 2 sqrt(2/pi) {3 * 0.044715, 1}
    } else if (act == FP8_ACT_SILU) {
        const float c = within(x, 200.0f);
        float s, ds;
        sigmoid2(c * 1.442695041f, &s, &ds);
        *f = (x < 0.0f ? c : x) * s;
        *d = fmaf(c, ds, s);
    } else if (act == FP8_ACT_RELU) {
        *f = x <= 0.0f ? 0.0f : x;
        *d = x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;
    } else {
        *f = x;
        *d = 1.0f;
    }
}

// Columns n .. n + W - 1 (nv of them valid) of row m: t the unscaled sums (with
// kEpiGlu the gate's, u the up projection's).  Every output is rounded once,
// from fp32.  The column sums of a backward epilogue are added to sa (with
// kEpiGluBwd: the gate's, sb the up projection's).
template <int MODE, int W>
__device__ __forceinline__ void epi_row(const Epi& e, int64_t m, int64_t n, int nv, float (&t)[W], float (&u)[W],
                                        float (&sa)[W], float (&sb)[W]) {
    float f, d, x[W], y[W];
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
