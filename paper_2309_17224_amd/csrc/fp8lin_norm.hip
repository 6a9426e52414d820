// Layer norm of the GPT models (Table 1), forward and backward, and the column
// sums that a bias gradient is, for gfx950.
//
//   h = x (+ res), rounded; y = (h - mean) rstd g + b, rstd = 1 / sqrt(var + eps)
//   dx = rstd (w - mean_j w - xh mean_j (w xh)) (+ dres), w = dy g, xh = (h - mean) rstd
//   dg = sum over rows of dy xh, db = sum over rows of dy
//
// Everything is bound by memory: h and dy are read once where a row fits the
// registers of its threads, statistics are fp32 and of the centred values (the
// mean is taken first), and each output is rounded once.  8192 x 5120 with residual and
// codes: 80 us, 4.7 TB/s, near the rate of a device copy (16384 x 4096 without them 5.1);
// backward of 4096 x 8192 with the residual's gradient 55 us, 4.9 TB/s, and 4 for the sums
// of its partial rows.  fp32: 8192 x 5120 76 us forward (4.4 TB/s), 113 backward (4.5).
// Backward beyond 8192 columns, two eights a thread: 4096 x 12288 96 us (3.1 TB/s), fp32 171;
// 21 and 26 registers are spilled there (7 of fp32 rows of 4097 columns and more).  Beyond
// 16384 rows are read again: 4096 x 20480 148 us forward, 224 backward (2.3).
#include <algorithm>

#include "fp8lin_glue.h"
#include "fp8lin_vals.h"

namespace fp8lin {
namespace {

// Threads that share a row, and eights of columns each of them holds.
constexpr int kNormBlock = 256;

// Sum over the T threads of a row, the same in all of them; red: a slot for
// every wave of the block, free again after the next barrier.
template <int T>
__device__ __forceinline__ float row_sum(float v, float* red) {
    v = wave_sum(v);
    if (T == 64) return v;
    const int w = threadIdx.x >> 6;
    __syncthreads();  // earlier sums have been read
    if ((threadIdx.x & 63) == 0) red[w] = v;
    __syncthreads();
    constexpr int kW = T / 64;
    const float* p = red + w / kW * kW;
    float s[kW];
#pragma unroll
    for (int i = 0; i < kW; ++i) s[i] = p[i];
#pragma unroll
    for (int d = 1; d < kW; d *= 2)
#pragma unroll
        for (int i = 0; i + d < kW; i += 2 * d) s[i] += s[i + d];
    return s[0];
}

// Two such sums in one exchange; red: two slots for every wave.
template <int T>
__device__ __forceinline__ void row_sum2(float& a, float& b, float2* red) {
    a = wave_sum(a);
    b = wave_sum(b);
    if (T == 64) return;
    const int w = threadIdx.x >> 6;
    __syncthreads();  // earlier sums have been read
    if ((threadIdx.x & 63) == 0) red[w] = make_float2(a, b);
    __syncthreads();
    constexpr int kW = T / 64;
    const float2* p = red + w / kW * kW;
    float2 s[kW];
#pragma unroll
    for (int i = 0; i < kW; ++i) s[i] = p[i];
#pragma unroll
    for (int d = 1; d < kW; d *= 2)
#pragma unroll
        for (int i = 0; i + d < kW; i += 2 * d) s[i].x += s[i + d].x, s[i].y += s[i + d].y;
    a = s[0].x;
    b = s[0].y;
}

// Eight values as they lie in memory, read once (the first nv of them; the rest 0).
template <int DT>
struct Raw8 {
    uint4 w[DT == FP8_DT_F32 ? 2 : 1];
};

template <int DT>
__device__ __forceinline__ Raw8<DT> ld_raw8(const void* base, int64_t at, int nv) {
    Raw8<DT> r;
    if (nv >= 8) {
#pragma unroll
        for (int k = 0; k < (DT == FP8_DT_F32 ? 2 : 1); ++k)
            r.w[k] = ld_stream((const char*)base + at * (DT == FP8_DT_F32 ? 4 : 2) + 16 * k);
    } else {
        float v[8];
        ld_vals<8>(base, at, DT, nv, v);
        if (DT == FP8_DT_F32) {
            r.w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            r.w[DT == FP8_DT_F32 ? 1 : 0] =
                make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
        } else {  // the upper halves, exact
            r.w[0] = make_uint4(__float_as_uint(v[0]) >> 16 | (__float_as_uint(v[1]) & 0xFFFF0000u),
                                __float_as_uint(v[2]) >> 16 | (__float_as_uint(v[3]) & 0xFFFF0000u),
                                __float_as_uint(v[4]) >> 16 | (__float_as_uint(v[5]) & 0xFFFF0000u),
                                __float_as_uint(v[6]) >> 16 | (__float_as_uint(v[7]) & 0xFFFF0000u));
        }
    }
    return r;
}

template <int DT>
__device__ __forceinline__ void values8(const Raw8<DT>& r, float (&v)[8]) {
    const uint32_t w[8] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w, r.w[DT == FP8_DT_F32 ? 1 : 0].x,
                           r.w[DT == FP8_DT_F32 ? 1 : 0].y, r.w[DT == FP8_DT_F32 ? 1 : 0].z, r.w[DT == FP8_DT_F32 ? 1 : 0].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = DT == FP8_DT_F32 ? __uint_as_float(w[i]) : i & 1 ? hi_f(w[i >> 1]) : lo_f(w[i >> 1]);
}

// One value of v rounded to type DT.
template <int DT>
__device__ __forceinline__ float rounded(float v) {
    return DT == FP8_DT_BF16 ? __uint_as_float(pack_bf16x2(v, 0.0f) << 16) : v;
}

// ------------------------------------------------------------- forward
// The sum over a row of what each of its T threads has in parts.  A wave that holds a row
// alone has a part for each wave of a block that would, and adds them in that block's
// order: a row's bits do not depend on how many rows there are.
template <int T, int G>
__device__ __forceinline__ float parts_sum(float (&v)[G], float* red) {
    if constexpr (G == 1) return row_sum<T>(v[0], red);
#pragma unroll
    for (int i = 0; i < G; ++i) v[i] = wave_sum(v[i]);
#pragma unroll
    for (int d = 1; d < G; d *= 2)
#pragma unroll
        for (int i = 0; i + d < G; i += 2 * d) v[i] += v[i + d];
    return v[0];
}

template <int DT, int T, int CH, int FMT>
__global__ __launch_bounds__(kNormBlock) void layernorm_kernel(NormArgs a, const int32_t* __restrict__ pred,
                                                               int32_t* __restrict__ used, uint32_t* __restrict__ parts,
                                                               uint8_t* __restrict__ q, int64_t ldq) {
    constexpr bool kQuant = FMT >= 0;
    __shared__ float red[kNormBlock / 64];
    __shared__ uint32_t redm[kNormBlock / 64];
    const int tid = threadIdx.x % T;
    const int64_t r = (int64_t)blockIdx.x * (kNormBlock / T) + threadIdx.x / T;
    const bool live = r < a.rows;
    const int64_t row = live ? r : a.rows - 1, cols = a.cols;
    const bool in_regs = cols <= (int64_t)8 * T * CH;
    constexpr int kParts = T > 64 ? 1 : CH < 4 ? CH : 4;
    const int bq = kQuant ? fused_bias(pred, used) : 0;
    float h[CH][8];
    auto sum_res = [&](const Raw8<DT>& x, const Raw8<DT>& y, float (&v)[8]) {
        values8(x, v);
        if (a.res) {
            float w[8];
            values8(y, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = rounded<DT>(v[i] + w[i]);
        }
    };
    auto load = [&](int64_t c, float (&v)[8]) {
        const int nv = (int)min((int64_t)8, cols - c);
        Raw8<DT> x = ld_raw8<DT>(a.x, row * a.ldx + c, nv), y{};
        if (a.res) y = ld_raw8<DT>(a.res, row * a.ldr + c, nv);
        sum_res(x, y, v);
    };
    float sum[kParts] = {};
    if (in_regs) {
        Raw8<DT> x[CH], y[CH];  // every load of the row under way before the first is used
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = (int64_t)8 * (tid + T * k);
            x[k] = y[k] = Raw8<DT>{};
            if (c < cols) x[k] = ld_raw8<DT>(a.x, row * a.ldx + c, (int)min((int64_t)8, cols - c));
        }
        if (a.res) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int64_t c = (int64_t)8 * (tid + T * k);
                if (c < cols) y[k] = ld_raw8<DT>(a.res, row * a.ldr + c, (int)min((int64_t)8, cols - c));
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            sum_res(x[k], y[k], h[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[k % kParts] += h[k][i];
        }
    } else {
        for (int64_t c = 8 * tid; c < cols; c += 8 * T) {
            float v[8];
            load(c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v[i];
        }
    }
    const float mean = parts_sum<T>(sum, red) / (float)cols;
    float ss[kParts] = {};
    auto centred = [&](int64_t c, const float (&v)[8], float& s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = c + i < cols ? v[i] - mean : 0.0f;
            s = fmaf(d, d, s);
        }
    };
    if (in_regs) {
#pragma unroll
        for (int k = 0; k < CH; ++k) centred((int64_t)8 * (tid + T * k), h[k], ss[k % kParts]);
    } else {
        for (int64_t c = 8 * tid; c < cols; c += 8 * T) {
            float v[8];
            load(c, v);
            centred(c, v, ss[0]);
        }
    }
    const float rstd = 1.0f / sqrtf(parts_sum<T>(ss, red) / (float)cols + a.eps);
    if (live && tid == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    const bool cast = kQuant && pred;
    uint32_t mag = 0;
    auto store = [&](int64_t c, const float (&v)[8]) {
        if (!live || c >= cols) return;
        const int nv = (int)min((int64_t)8, cols - c);
        if (a.h) st_vals<8>(a.h, r * a.ldh + c, DT, nv, v);
        float g[8], b[8] = {}, y[8];
        ld_vals<8>(a.g, c, a.g_dt, nv, g);
        if (a.b) ld_vals<8>(a.b, c, a.g_dt, nv, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaf((v[i] - mean) * rstd, g[i], b[i]);
        st_vals<8>(a.y, r * a.ldy + c, DT, nv, y);
        if (kQuant) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = i < nv ? y[i] : 0.0f;
            const uint4 w = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                                       pack_bf16x2(y[6], y[7]));
            mag = max(mag, mag8(w));
            if (cast) {
                const uint2 c8 = codes8<FMT < 0 ? 0 : FMT>(w, bq);
                uint8_t* p = q + r * ldq + c;
                // (plain stores: 8192 x 5120 65.9 us, 1000 x 8192 14.6; so 64.6, 13.6)
                if (nv == 8) __builtin_nontemporal_store((u32x2_any{c8.x, c8.y}), (u32x2_any*)p);
                else
                    for (int i = 0; i < nv; ++i) p[i] = (uint8_t)((i < 4 ? c8.x : c8.y) >> (8 * (i & 3)));
            }
        }
    };
    if (in_regs) {
#pragma unroll
        for (int k = 0; k < CH; ++k) store((int64_t)8 * (tid + T * k), h[k]);
    } else {
        for (int64_t c = 8 * tid; c < cols; c += 8 * T) {
            float v[8];
            load(c, v);
            store(c, v);
        }
    }
    if (kQuant) {
        const uint32_t bm = block_max(mag, redm);
        if (threadIdx.x == 0) parts[blockIdx.x] = bm;
    }
}

// ------------------------------------------------------------- backward
// A row's threads hold its columns and, of every row they take, add their part
// of the column sums: one row of part for each workgroup, its groups of T threads added in
// order.  CH == 0: rows
// too wide for that, read twice, and the column sums are colsum_kernel's.
template <int DT, int T, int CH>
__global__ __launch_bounds__(T < kNormBlock ? kNormBlock : T) void layernorm_bwd_kernel(NormArgs a, float* __restrict__ part) {
    // Two eights a thread leave no registers for the next row or the gain.
    constexpr bool kAhead = CH <= 1;
    constexpr int kBlock = T < kNormBlock ? kNormBlock : T, kCh = CH > 0 ? CH : 1;
    __shared__ float2 red[kBlock / 64];
    const int tid = threadIdx.x % T;
    const int64_t slot = (int64_t)blockIdx.x * (kBlock / T) + threadIdx.x / T, slots = (int64_t)gridDim.x * (kBlock / T);
    const int64_t cols = a.cols;
    const float inv = 1.0f / (float)cols;
    float g[8] = {}, sg[kCh][8], sb[kCh][8];
    auto gain = [&](int k) {
        const int64_t c = (int64_t)8 * (tid + T * k);
        if (c < cols) ld_vals<8>(a.g, c, a.g_dt, (int)min((int64_t)8, cols - c), g);
    };
#pragma unroll
    for (int k = 0; k < kCh; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sg[k][i] = sb[k][i] = 0.0f;
    if (CH == 1) gain(0);
    // every thread of a block takes the same number of turns (the sums are the block's)
    const int64_t turns = (a.rows - (int64_t)blockIdx.x * (kBlock / T) + slots - 1) / slots;
    // what a row needs, one row ahead: while a row's sums go round the block, the next
    // row is on its way
    Raw8<DT> xr[kCh], dr[kCh], er[kCh];
    float mean = 0.0f, rstd = 0.0f, mean_n = 0.0f, rstd_n = 0.0f;
    auto row_of = [&](int64_t turn) { return min(slot + turn * slots, a.rows - 1); };
    auto ahead = [&](int64_t turn) {
        const int64_t row = row_of(turn);
        mean_n = a.mean[row];
        rstd_n = a.rstd[row];
        if (CH == 0) return;
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
            const int64_t c = (int64_t)8 * (tid + T * k);
            const int nv = (int)min((int64_t)8, cols - c);
            xr[k] = dr[k] = er[k] = Raw8<DT>{};
            if (c < cols) {
                xr[k] = ld_raw8<DT>(a.x, row * a.ldx + c, nv);
                dr[k] = ld_raw8<DT>(a.dy, row * a.lddy + c, nv);
                if (kAhead && a.dres) er[k] = ld_raw8<DT>(a.dres, row * a.lddr + c, nv);
            }
        }
    };
    if (kAhead) ahead(0);
    for (int64_t turn = 0; turn < turns; ++turn) {
        const int64_t r = slot + turn * slots, row = row_of(turn);
        const bool live = r < a.rows;
        if (!kAhead) ahead(turn);
        mean = mean_n;
        rstd = rstd_n;
        float xh[kCh][8], dy[kCh][8], c1 = 0.0f, c2 = 0.0f;
        Raw8<DT> e[kCh];
        auto finish = [&](int64_t c, const float (&x)[8], const float (&d)[8], const float (&gg)[8], const Raw8<DT>& ee) {
            if (!live || c >= cols) return;
            float y[8], w[8];
            values8(ee, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = rstd * (d[i] * gg[i] - c1 - x[i] * c2);
                if (a.dres) y[i] += w[i];
            }
            st_vals<8>(a.y, r * a.ldy + c, DT, (int)min((int64_t)8, cols - c), y);
        };
        auto centre = [&](const Raw8<DT>& x, const Raw8<DT>& d, int nv, float (&xv)[8], float (&dv)[8]) {
            values8(x, xv);
            values8(d, dv);
#pragma unroll
            for (int i = 0; i < 8; ++i) xv[i] = i < nv ? (xv[i] - mean) * rstd : 0.0f;
        };
        if (CH > 0) {
#pragma unroll
            for (int k = 0; k < kCh; ++k) {
                centre(xr[k], dr[k], (int)min((int64_t)8, cols - (int64_t)8 * (tid + T * k)), xh[k], dy[k]);
                e[k] = er[k];
            }
            if (kAhead && turn + 1 < turns) ahead(turn + 1);
#pragma unroll
            for (int k = 0; k < kCh; ++k) {
                if (CH > 1) gain(k);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float w = dy[k][i] * g[i];
                    c1 += w;
                    c2 = fmaf(w, xh[k][i], c2);
                    if (live) {
                        sg[k][i] = fmaf(dy[k][i], xh[k][i], sg[k][i]);
                        sb[k][i] += dy[k][i];
                    }
                }
            }
        } else {
            if (turn + 1 < turns) ahead(turn + 1);
            for (int64_t c = 8 * tid; c < cols; c += 8 * T) {
                const int nv = (int)min((int64_t)8, cols - c);
                float gg[8];
                centre(ld_raw8<DT>(a.x, row * a.ldx + c, nv), ld_raw8<DT>(a.dy, row * a.lddy + c, nv), nv, xh[0], dy[0]);
                ld_vals<8>(a.g, c, a.g_dt, nv, gg);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float w = dy[0][i] * gg[i];
                    c1 += w;
                    c2 = fmaf(w, xh[0][i], c2);
                }
            }
        }
        row_sum2<T>(c1, c2, red);
        c1 *= inv;
        c2 *= inv;
        if (CH > 0) {
#pragma unroll
            for (int k = 0; k < kCh; ++k) {
                if (CH > 1) {
                    gain(k);
                    const int64_t c = (int64_t)8 * (tid + T * k);
                    if (a.dres && c < cols) e[k] = ld_raw8<DT>(a.dres, row * a.lddr + c, (int)min((int64_t)8, cols - c));
                }
                finish((int64_t)8 * (tid + T * k), xh[k], dy[k], g, e[k]);
            }
        } else {
            for (int64_t c = 8 * tid; c < cols; c += 8 * T) {
                const int nv = (int)min((int64_t)8, cols - c);
                float gg[8];
                Raw8<DT> ee{};
                centre(ld_raw8<DT>(a.x, row * a.ldx + c, nv), ld_raw8<DT>(a.dy, row * a.lddy + c, nv), nv, xh[0], dy[0]);
                if (a.dres) ee = ld_raw8<DT>(a.dres, row * a.lddr + c, nv);
                ld_vals<8>(a.g, c, a.g_dt, nv, gg);
                finish(c, xh[0], dy[0], gg, ee);
            }
        }
    }
    if (CH > 0 && part) {
        constexpr int kGroups = kBlock / T;
        if constexpr (kGroups > 1) {
            __shared__ float sums[kGroups - 1][16][T];
            const int grp = threadIdx.x / T;
            if (grp > 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[grp - 1][i][tid] = sg[0][i], sums[grp - 1][8 + i][tid] = sb[0][i];
            }
            __syncthreads();
            if (grp > 0) return;
#pragma unroll
            for (int k = 0; k < kGroups - 1; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) sg[0][i] += sums[k][i][tid], sb[0][i] += sums[k][8 + i][tid];
        }
        float* p = part + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
            const int64_t c = (int64_t)8 * (tid + T * k);
            const int nv = (int)max((int64_t)0, min((int64_t)8, cols - c));
            st_vals<8>(p, c, FP8_DT_F32, nv, sg[k]);
            st_vals<8>(p, cols + c, FP8_DT_F32, nv, sb[k]);
        }
    }
}

// ------------------------------------------------------------- column sums
// A workgroup sums 512 columns over `per` consecutive rows, a wave each fourth row,
// eight rows' loads at a time; its waves' sums are added in order: one row of part for
// each blockIdx.y.  With one group of rows in all, the result itself goes to out0, out1
// (of type out_dt; either may be null).  NORM: the layer norm's two sums, of dy xh into
// columns [0, cols) (out0) and dy into [cols, 2 cols) (out1).
template <int DT, bool NORM>
__global__ __launch_bounds__(256) void colsum_kernel(NormArgs a, int64_t per, float* __restrict__ part, void* out0,
                                                     void* out1, int out_dt) {
    constexpr int kNs = NORM ? 2 : 1, kDepth = NORM ? 4 : 8;
    __shared__ float red[kNs][4][512];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 512 + 8 * lane;
    const int nv = (int)max((int64_t)0, min((int64_t)8, a.cols - c));
    float s[kNs][8] = {};
    if (nv > 0) {
        const int64_t end = min(((int64_t)blockIdx.y + 1) * per, a.rows);
        for (int64_t r0 = (int64_t)blockIdx.y * per + w; r0 < end; r0 += 4 * kDepth) {
            Raw8<DT> d[kDepth], x[kDepth];
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int64_t r = min(r0 + 4 * k, a.rows - 1);
                d[k] = ld_raw8<DT>(a.dy, r * a.lddy + c, nv);
                if (NORM) x[k] = ld_raw8<DT>(a.x, r * a.ldx + c, nv);
            }
#pragma unroll
            for (int k = 0; k < kDepth; ++k) {
                const int64_t r = r0 + 4 * k;
                if (r >= end) break;
                float dv[8], xv[8];
                values8(d[k], dv);
                if (NORM) {
                    values8(x[k], xv);
                    const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[0][i] = fmaf(dv[i], (xv[i] - mean) * rstd, s[0][i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) s[kNs - 1][i] += dv[i];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kNs; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) red[k][w][8 * lane + i] = s[k][i];
    __syncthreads();
    for (int i = threadIdx.x; i < 512; i += 256) {
        const int64_t col = (int64_t)blockIdx.x * 512 + i;
        if (col >= a.cols) break;
#pragma unroll
        for (int k = 0; k < kNs; ++k) {
            const float v = (red[k][0][i] + red[k][1][i]) + (red[k][2][i] + red[k][3][i]);
            if (gridDim.y > 1) {
                part[(int64_t)blockIdx.y * kNs * a.cols + k * a.cols + col] = v;
            } else if (void* out = k ? out1 : out0) {
                if (out_dt == FP8_DT_BF16) ((uint16_t*)out)[col] = (uint16_t)(pack_bf16x2(v, 0.0f) & 0xFFFFu);
                else ((float*)out)[col] = v;
            }
        }
    }
}

// The sums of few rows in one launch: 64 columns a workgroup at a time, 128 rows at a time over
// its 1024 threads, all of up to four such loads under way; then over the lanes and waves
// in a fixed order.
constexpr int64_t kFewRows = 1024;
template <int DT>
__global__ __launch_bounds__(1024) void colsum_few_kernel(const void* __restrict__ x, int64_t rows, int64_t cols,
                                                          int64_t ldx, void* __restrict__ out, int out_dt) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < cols; c0 += (int64_t)gridDim.x * 64) {
        const int64_t c = c0 + 8 * (lane & 7);
        const int nv = (int)max((int64_t)0, min((int64_t)8, cols - c));
        float s[8] = {};
        for (int64_t r0 = 8 * w + (lane >> 3); r0 < rows; r0 += 512) {
            Raw8<DT> v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = Raw8<DT>{};
                if (nv > 0 && r0 + 128 * k < rows) v[k] = ld_raw8<DT>(x, (r0 + 128 * k) * ldx + c, nv);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float f[8];
                values8(v[k], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] += f[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int off = 8; off < 64; off <<= 1) s[i] += __shfl_xor(s[i], off, 64);
            if (lane < 8) red[w][8 * lane + i] = s[i];
        }
        __syncthreads();
        const int64_t col = c0 + lane;
        if (w == 0 && col < cols) {
            float v = red[0][lane];
#pragma unroll
            for (int k = 1; k < 16; ++k) v += red[k][lane];
            if (out_dt == FP8_DT_BF16) ((uint16_t*)out)[col] = (uint16_t)(pack_bf16x2(v, 0.0f) & 0xFFFFu);
            else ((float*)out)[col] = v;
        }
        __syncthreads();  // red may be written again
    }
}

// ------------------------------------------------------------- host side
constexpr int64_t kMaxNormBlocks = 1 << 23;  // of a launch
constexpr int64_t kNormWidest = 16384;  // columns a row's threads hold in the backward pass

// Rows of a group of colsum_kernel: about 1024 workgroups, groups of 16 rows (four to a
// wave) at least.  A turn of 32 rows (16 of the layer norm's sums) past a group's end is loaded and not
// added: of 4096 x 5120 64 rows for the 41 of a group (15.1 us with the second launch, 2.8
// TB/s; 8192 x 4096, 64 for 64, 18.1 us, 3.7).
int64_t sum_group(int64_t rows, int64_t cols) {
    const int64_t wide = (cols + 511) / 512, groups = std::max<int64_t>(1, std::min<int64_t>(256, 1024 / wide));
    return std::max<int64_t>(16, (rows + groups - 1) / groups);
}

// Threads of a row in the backward pass: 8 columns each, 16 beyond 8192.
int bwd_threads(int64_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024; }

int64_t bwd_blocks(int64_t rows, int64_t cols) {
    // Every block leaves a row of partial sums, which bounds them: blocks of up to four rows
    // at a time are small enough for two on a compute unit, each hiding the other's
    // exchanges (16384 x 1024 in 256, 512 and 1024 of them: 41.7, 26.8, 27.4 us; 4096 x 2048
    // 25.0, 19.8, 25.0), with at least two rows one after another; of wider rows one
    // (8192 x 5120 in 256 and 512: 62.5, 66.8; 2000 x 4096 18.0, 21.9; 16384 x 4096 81.3, 77.8).
    const int t = bwd_threads(cols), per = t < kNormBlock ? kNormBlock / t : 1;
    const int64_t all = (rows + per - 1) / per;
    return t <= kNormBlock ? std::min<int64_t>((all + 1) / 2, 512) : std::min<int64_t>(all, 256);
}

}  // namespace

int64_t colsum_rows(int64_t rows, int64_t cols) {
    const int64_t per = sum_group(rows, cols);
    return (rows + per - 1) / per;
}

int64_t norm_sum_rows(int64_t rows, int64_t cols) {
    if (cols > kNormWidest) return colsum_rows(rows, cols);
    return bwd_blocks(rows, cols);
}

int32_t launch_layernorm(const NormArgs& a, const FusedQuant* fq, hipStream_t s) {
    const bool quant = fq && fq->q;
    int64_t grid = 0;
    int32_t st = FP8_OK;
    auto go = [&](auto D, auto Tt, auto C, auto Fm) {
        constexpr int kT = decltype(Tt)::value;
        constexpr int64_t kPer = kNormBlock / kT;
        grid = (a.rows + kPer - 1) / kPer;
        // (a launch has fewer than 2^32 threads)
        for (int64_t b0 = 0; b0 < grid && st == FP8_OK; b0 += kMaxNormBlocks) {
            const int64_t r0 = b0 * kPer, nb = std::min(grid - b0, kMaxNormBlocks), size = decltype(D)::value == FP8_DT_F32 ? 4 : 2;
            NormArgs p = a;
            p.rows = std::min(a.rows - r0, nb * kPer);
            p.x = (const char*)a.x + r0 * a.ldx * size;
            p.y = (char*)a.y + r0 * a.ldy * size;
            if (a.res) p.res = (const char*)a.res + r0 * a.ldr * size;
            if (a.h) p.h = (char*)a.h + r0 * a.ldh * size;
            if (a.mean) p.mean = a.mean + r0;
            if (a.rstd) p.rstd = a.rstd + r0;
            hipLaunchKernelGGL((layernorm_kernel<decltype(D)::value, kT, decltype(C)::value, decltype(Fm)::value>),
                               dim3((unsigned)nb), dim3(kNormBlock), 0, s, p, quant ? fq->pred : nullptr,
                               quant ? (int32_t*)fq->ws : nullptr, quant ? fq->ws + 1 + b0 : nullptr,
                               quant ? fq->q + r0 * fq->ldq : nullptr, quant ? fq->ldq : (int64_t)0);
            st = hip_status();
        }
    };
    auto size = [&](auto D, auto Fm) {
        // A wave for a row needs no exchange in LDS and no barrier, which counts where rows
        // queue for the compute units; a block for a row has the shorter way through it.
        // Plain and with codes, us: 64 x 768 by a wave 4.0, 7.4, by a block 3.6, 6.6; 4096 x
        // 768 5.6, 9.7 and 9.0, 14.7; 1000 x 1283 6.5, 10.4 and 5.3, 8.8; 2000 x 1283 7.6,
        // 11.4 and 7.4, 12.7; 8192 x 1283 17.5, 25.8 and 21.8, 35.3; 8192 x 2560 21.4, 34.4
        // and 22.5, 43.0; 8192 x 4096 26.8, 47.6 and 28.5, 48.4, with a residual 43.4 and 40.8.
        // The borders lie between these sizes; nearer to them the two were not measured.
        if (a.cols <= 512) go(D, IC<64>{}, IC<1>{}, Fm);
        else if (a.cols <= 1024 && a.rows > 768) go(D, IC<64>{}, IC<2>{}, Fm);
        else if (a.cols <= 2048 && a.rows >= 2000) go(D, IC<64>{}, IC<4>{}, Fm);
        else if (a.cols <= 2048) go(D, IC<256>{}, IC<1>{}, Fm);
        else if (a.cols <= 2560 && a.rows >= 3000) go(D, IC<64>{}, IC<8>{}, Fm);
        else if (a.cols <= 4096) go(D, IC<256>{}, IC<2>{}, Fm);
        else if (a.cols <= 8192) go(D, IC<256>{}, IC<4>{}, Fm);
        else go(D, IC<256>{}, IC<8>{}, Fm);
    };
    if (a.dt == FP8_DT_F32) size(IC<FP8_DT_F32>{}, IC<-1>{});
    else if (!quant) size(IC<FP8_DT_BF16>{}, IC<-1>{});
    else with_fmt(fq->fmt, [&](auto Fm) { size(IC<FP8_DT_BF16>{}, Fm); });
    if (st != FP8_OK || !quant) return st;
    return launch_quant_check(a.y, FP8_DT_BF16, a.rows, a.cols, a.ldy, fq->fmt, fq->margin, fq->ws + 1, (int)grid,
                              (const int32_t*)fq->ws, fq->bias, fq->amax_bits, fq->flags, fq->q, fq->ldq, nullptr, 0, s);
}

int32_t launch_layernorm_bwd(const NormArgs& a, float* dg, float* db, float* part, hipStream_t s) {
    const int64_t sums = norm_sum_rows(a.rows, a.cols);
    const bool want = dg || db;
    auto go = [&](auto D, auto Tt, auto C) {
        constexpr int kT = decltype(Tt)::value;
        const int64_t blocks = decltype(C)::value == 0 ? std::min<int64_t>(a.rows, 2048) : bwd_blocks(a.rows, a.cols);
        hipLaunchKernelGGL((layernorm_bwd_kernel<decltype(D)::value, kT, decltype(C)::value>), dim3((unsigned)blocks),
                           dim3(kT < kNormBlock ? kNormBlock : kT), 0, s, a, want ? part : nullptr);
    };
    auto size = [&](auto D) {
        switch (bwd_threads(a.cols)) {
            case 64: go(D, IC<64>{}, IC<1>{}); break;
            case 128: go(D, IC<128>{}, IC<1>{}); break;
            case 256: go(D, IC<256>{}, IC<1>{}); break;
            case 512: go(D, IC<512>{}, IC<1>{}); break;
            default:
                if (a.cols <= 8192) go(D, IC<1024>{}, IC<1>{});
                else if (a.cols <= kNormWidest) go(D, IC<1024>{}, IC<2>{});
                else go(D, IC<1024>{}, IC<0>{});
        }
    };
    if (a.dt == FP8_DT_BF16) size(IC<FP8_DT_BF16>{});
    else size(IC<FP8_DT_F32>{});
    int32_t st = hip_status();
    if (st != FP8_OK || !want) return st;
    if (a.cols > kNormWidest) {
        const dim3 grid((unsigned)((a.cols + 511) / 512), (unsigned)sums);
        const int64_t per = sum_group(a.rows, a.cols);
        if (a.dt == FP8_DT_BF16)
            hipLaunchKernelGGL((colsum_kernel<FP8_DT_BF16, true>), grid, dim3(256), 0, s, a, per, part, dg, db, FP8_DT_F32);
        else
            hipLaunchKernelGGL((colsum_kernel<FP8_DT_F32, true>), grid, dim3(256), 0, s, a, per, part, dg, db, FP8_DT_F32);
        st = hip_status();
        if (st != FP8_OK || sums == 1) return st;
    }
    return launch_sums_finish(part, sums, 2 * a.cols, dg, a.cols, db, FP8_DT_F32, s);
}

int32_t launch_colsum(const void* x, int dt, int64_t rows, int64_t cols, int64_t ldx, void* out, int out_dt, float* part,
                      hipStream_t s) {
    if (rows <= kFewRows) {
        const dim3 grid((unsigned)sum_blocks(cols));
        if (dt == FP8_DT_BF16)
            hipLaunchKernelGGL((colsum_few_kernel<FP8_DT_BF16>), grid, dim3(1024), 0, s, x, rows, cols, ldx, out, out_dt);
        else
            hipLaunchKernelGGL((colsum_few_kernel<FP8_DT_F32>), grid, dim3(1024), 0, s, x, rows, cols, ldx, out, out_dt);
        return hip_status();
    }
    NormArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.dy = x;
    a.lddy = ldx;
    const int64_t sums = colsum_rows(rows, cols);
    const dim3 grid((unsigned)((cols + 511) / 512), (unsigned)sums);
    const int64_t per = sum_group(rows, cols);
    void* none = nullptr;
    if (dt == FP8_DT_BF16)
        hipLaunchKernelGGL((colsum_kernel<FP8_DT_BF16, false>), grid, dim3(256), 0, s, a, per, part, out, none, out_dt);
    else
        hipLaunchKernelGGL((colsum_kernel<FP8_DT_F32, false>), grid, dim3(256), 0, s, a, per, part, out, none, out_dt);
    const int32_t st = hip_status();
    if (st != FP8_OK || sums == 1) return st;
    return launch_sums_finish(part, sums, cols, out, cols, nullptr, out_dt, s);
}

}  // namespace fp8lin
