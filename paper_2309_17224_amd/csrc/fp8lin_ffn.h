// The matmuls of a feed-forward block with what follows them in the epilogue, for
// gfx950: bias, activation and residual sum (GPT), the gated pair of projections
// (Llama 2), and in the backward pass the slope of the activation and the bias
// gradient.
//
//   kEpiAct     y = act(s x w + bias) + res             s = 2^-(b_a + b_b) (Eq. 2)
//   kEpiGlu     a = act(g) u, (g | u) = s x (wg | wu) + bias
//   kEpiActBwd  dz = t act'(z), t = s dy w^T; sum over rows
//   kEpiGluBwd  dg = t u act'(g), du = t act(g); sums over rows
//
// The main loops are those of the plain matmuls (fp8lin_gemm.hip, _stream,
// _ragged), and so is the choice among them.  The gated pair multiplies A by
// both matrices in one tile whose B rows are blocks of 16 from them in turn, so
// that one lane ends with the same columns of both products.
// The sums go through LDS, 32 rows of a wave at a time, so that a lane gets eight
// consecutive columns of one row: every global access is then a 16-byte piece of
// a row run, and the epilogue's code exists once, in a loop.
#pragma once

#include "fp8lin_epilogue.h"
#include "fp8lin_glue.h"
#include "fp8lin_mm_256.h"
#include "fp8lin_mm_ragged.h"

namespace fp8lin {
namespace {

constexpr int pow2_up(int n) { return n <= 1 ? 1 : 2 * pow2_up((n + 1) / 2); }

// Geometry of a wave's epilogue: MBLK x NBLK blocks of 16 x 16 sums, staged 32 rows
// at a time; an eight of columns to a lane, kNp consecutive rows of it one after
// another (so that their codes' bytes end in one lane for the transposed copy).
template <int MODE, int NBLK>
struct EpiGeo {
    static constexpr bool kPair = MODE == kEpiGlu;
    static constexpr int kRow = NBLK * 64 + 16;           // staging row, bytes
    static constexpr int kOct = kPair ? NBLK : 2 * NBLK;  // eights of columns in a row
    static constexpr int kLpr = pow2_up(kOct), kNp = kLpr / 2;  // lanes a row, rows of a lane
    static_assert((!kPair || NBLK % 2 == 0) && kLpr <= 16 && kNp >= 1, "blocks of a wave");
};

// Stages rows 32 i2 .. 32 i2 + 31 of a wave's sums, unscaled by 2^sh.
template <int I2, int MBLK, int NBLK>
__device__ __forceinline__ void stage_sums(uint8_t* ep, const v4f (&acc)[MBLK][NBLK], int sh) {
    constexpr int kRow = NBLK * 64 + 16;
    const int lane = threadIdx.x & 63, frow = lane & 15, fg = lane >> 4;
#pragma unroll
    for (int ii = 0; ii < 2; ++ii)
#pragma unroll
        for (int j = 0; j < NBLK; ++j) {
            const v4f a = acc[2 * I2 + ii][j];
            *(float4*)(ep + (ii * 16 + frow) * kRow + (j * 16 + 4 * fg) * 4) =
                make_float4(ldexpf(a[0], sh), ldexpf(a[1], sh), ldexpf(a[2], sh), ldexpf(a[3], sh));
        }
}

__device__ __forceinline__ void unpack8(uint4 w, float (&v)[8]) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x[i] << 16);
        v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
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

// The codes c of NP consecutive rows (rows of them in the matrix) of eight columns
// to the transposed copy: eight runs of NP bytes, ld apart.
template <int NP>
__device__ __forceinline__ void store_transposed(uint8_t* p, int64_t ld, const uint2 (&c)[NP], int rows) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t t[(NP + 3) / 4][4];
#pragma unroll
        for (int g = 0; g < (NP + 3) / 4; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) t[g][i] = 4 * g + i < NP ? (h ? c[(4 * g + i) % NP].y : c[(4 * g + i) % NP].x) : 0u;
            transpose4(t[g]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint8_t* q = p + (4 * h + i) * ld;
            if (NP == 8 && rows >= 8) {
                st8_any(q, t[0][i], t[(NP + 3) / 4 - 1][i]);
            } else if (NP == 4 && rows >= 4) {
                *(u32_any*)q = t[0][i];
            } else {
#pragma unroll
                for (int r = 0; r < NP; ++r)
                    if (r < rows) q[r] = (uint8_t)(t[r >> 2][i] >> (8 * (r & 3)));
            }
        }
    }
}

// One half (32 rows) of a wave's epilogue where every lane's eight columns are
// all in the matrix (active) or all outside and the output is bf16.  zb, kb, ob, ..:
// the wave's first element in each tensor (uniform), so that the lanes' offsets are
// 32-bit.  rows: rows of the wave in the matrix (> 0).  What is read from memory is
// under way before the sums are staged.
template <int MODE, int ACT, int I2, int MBLK, int NBLK>
__device__ __forceinline__ void half_epilogue(const Epi& e, uint8_t* ep, const v4f (&acc)[MBLK][NBLK], int64_t m0, int64_t n0,
                                              int rows, bool active, int sh, int bq, const float (&ba)[8],
                                              const float (&bu)[8], float (&sa)[8], float (&sb)[8], uint32_t& mag) {
    using G = EpiGeo<MODE, NBLK>;
    constexpr bool kPair = G::kPair, kTwo = MODE == kEpiGluBwd;
    constexpr int kNp = G::kNp, kFmt = epi_fwd(MODE) ? FP8_E4M3 : FP8_E5M2;
    const int lane = threadIdx.x & 63, oct = lane & (G::kLpr - 1), r0 = lane / G::kLpr * kNp;
    const uint32_t col = 8 * oct;
    uint4 pre[kNp], pre2[kTwo ? kNp : 1];
    const bool res = MODE == kEpiAct && e.res;
    if (active && (!epi_fwd(MODE) || res)) {
        const uint16_t* src = MODE == kEpiAct ? (const uint16_t*)e.res : e.z;
        const uint32_t ld = (uint32_t)(MODE == kEpiAct ? e.ldres : e.ldz);
        src += m0 * ld + n0;
#pragma unroll
        for (int p = 0; p < kNp; ++p) {
            const uint32_t at = (uint32_t)min(32 * I2 + r0 + p, rows - 1) * ld + col;
            pre[p] = ld16_any(src + at);
            if (kTwo) pre2[p] = ld16_any(src + e.N + at);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    stage_sums<I2>(ep, acc, sh);
    if (!active) return;
    const uint8_t* src = ep + r0 * G::kRow + (kPair ? (oct >> 1) * 128 + (oct & 1) * 32 : oct * 32);
    float4 nx[kPair ? 4 : 2];
    auto fetch = [&](int p) {
        nx[0] = *(const float4*)(src + p * G::kRow);
        nx[1] = *(const float4*)(src + p * G::kRow + 16);
        if (kPair) {
            nx[kPair ? 2 : 0] = *(const float4*)(src + p * G::kRow + 64);
            nx[kPair ? 3 : 1] = *(const float4*)(src + p * G::kRow + 80);
        }
    };
    fetch(0);
    uint16_t* ob = (uint16_t*)e.out + m0 * e.ldo + n0;
    uint16_t* kb = e.keep + m0 * e.ldkeep + n0;
    uint8_t* qb = e.q + m0 * e.ldq + n0;
    uint2 c8[kNp], c8b[kTwo ? kNp : 1];
#pragma unroll
    for (int p = 0; p < kNp; ++p) {
        float t[8] = {nx[0].x, nx[0].y, nx[0].z, nx[0].w, nx[1].x, nx[1].y, nx[1].z, nx[1].w}, u[8], x[8], y[8], f, d;
        if (kPair) {
            const float4 a = nx[kPair ? 2 : 0], b = nx[kPair ? 3 : 1];
            const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = v[i];
        }
        if (p + 1 < kNp) fetch(p + 1);
        const int r = 32 * I2 + r0 + p;
        const bool in = r < rows;
        uint4 w, w2 = make_uint4(0u, 0u, 0u, 0u);
        if (epi_fwd(MODE)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[i] += ba[i];
                if (kPair) u[i] += bu[i];
            }
            if (e.keep) {
                w = pack8(t);
                if (kPair) w2 = pack8(u);
                if (in) {
                    st_stream(kb + ((uint32_t)r * (uint32_t)e.ldkeep + col), w);
                    if (kPair) st_stream(kb + e.N + ((uint32_t)r * (uint32_t)e.ldkeep + col), w2);
                }
            }
            if (res) unpack8(pre[p], x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                act_t<ACT>(t[i], &f, &d);
                y[i] = kPair ? f * u[i] : res ? f + x[i] : f;
            }
        } else {
            unpack8(pre[p], x);
            if (kTwo) unpack8(pre2[kTwo ? p : 0], u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                act_t<ACT>(x[i], &f, &d);
                if (kTwo) x[i] = t[i] * f;
                y[i] = (kTwo ? t[i] * u[i] : t[i]) * d;
            }
            if (e.sums && in) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sa[i] += y[i];
                    if (kTwo) sb[i] += x[i];
                }
            }
            if (kTwo) w2 = pack8(x);
        }
        w = pack8(y);
        if (in) {
            st_stream(ob + ((uint32_t)r * (uint32_t)e.ldo + col), w);
            if (kTwo) st_stream(ob + e.N + ((uint32_t)r * (uint32_t)e.ldo + col), w2);
        }
        if (e.q) {
            c8[p] = codes8<kFmt>(w, bq);
            if (in) mag = max(mag, mag8(w));
            if (in) st8_any(qb + ((uint32_t)r * (uint32_t)e.ldq + col), c8[p].x, c8[p].y);
            if (kTwo) {
                if (in) mag = max(mag, mag8(w2));
                c8b[kTwo ? p : 0] = codes8<kFmt>(w2, bq);
                if (in) st8_any(qb + e.N + ((uint32_t)r * (uint32_t)e.ldq + col), c8b[kTwo ? p : 0].x, c8b[kTwo ? p : 0].y);
            }
        }
    }
    if (e.q && e.qT) {
        uint8_t* q = e.qT + n0 * e.ldqT + m0 + ((uint32_t)(8 * oct) * (uint32_t)e.ldqT + 32 * I2 + r0);
        store_transposed<kNp>(q, e.ldqT, c8, rows - (32 * I2 + r0));
        if constexpr (kTwo) store_transposed<kNp>(q + e.N * e.ldqT, e.ldqT, c8b, rows - (32 * I2 + r0));
    }
}

// The epilogue of one wave: MBLK x NBLK blocks of 16 x 16 sums (laid out as in
// mm256_loop) of rows m0 .., columns n0 .. of the output (with kEpiGlu NBLK / 2
// blocks of columns of each projection); ep: 32 rows of LDS of its own; srow: its
// row of the column sums.  ACT < 0: the activation is e.act, and the epilogue exists
// once, in a loop (tiles cut by the matrix's last columns, any K).  Returns the
// largest output magnitude (bf16 pattern) where codes are written.
template <int MODE, int ACT, int MBLK, int NBLK>
__device__ __forceinline__ uint32_t wave_epilogue(const Epi& e, uint8_t* ep, const v4f (&acc)[MBLK][NBLK], int64_t m0,
                                                  int64_t n0, int64_t srow, int bq) {
    using G = EpiGeo<MODE, NBLK>;
    static_assert(MBLK == 2 || MBLK == 4, "halves of a wave");
    const int lane = threadIdx.x & 63;
    const int sh = -(*e.ba + *e.bb);
    const int oct = lane & (G::kLpr - 1), r0 = lane / G::kLpr * G::kNp;
    const int64_t n = n0 + 8 * oct;
    const int nv = oct < G::kOct ? (int)min((int64_t)8, e.N - n) : 0;
    const int rows = (int)min((int64_t)(16 * MBLK), e.M - m0);
    float sa[8] = {}, sb[8] = {};
    uint32_t mag = 0;
    if (ACT >= 0 && e.fast && !__any(nv > 0 && nv < 8)) {
        float ba[8] = {}, bu[8] = {};
        if (epi_fwd(MODE) && e.bias && nv > 0) {
            ld_vals<8>(e.bias, n, e.bias_dt, 8, ba);
            if (MODE == kEpiGlu) ld_vals<8>(e.bias, e.N + n, e.bias_dt, 8, bu);
        }
        if (rows > 0) {
            constexpr int kA = ACT >= 0 ? ACT : 0;
            half_epilogue<MODE, kA, 0>(e, ep, acc, m0, n0, rows, nv > 0, sh, bq, ba, bu, sa, sb, mag);
            if constexpr (MBLK == 4) half_epilogue<MODE, kA, 1>(e, ep, acc, m0, n0, rows, nv > 0, sh, bq, ba, bu, sa, sb, mag);
        }
    } else {
        const uint8_t* src = ep + r0 * G::kRow + (G::kPair ? (oct >> 1) * 128 + (oct & 1) * 32 : oct * 32);
        auto half = [&](int i2) {
#pragma unroll 1
            for (int p = 0; p < G::kNp; ++p) {
                const int r = 32 * i2 + r0 + p;
                if (nv <= 0 || r >= rows) continue;
                const float4 t0 = *(const float4*)(src + p * G::kRow), t1 = *(const float4*)(src + p * G::kRow + 16);
                float t[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w}, u[8];
                if (G::kPair) {
                    const float4 u0 = *(const float4*)(src + p * G::kRow + 64), u1 = *(const float4*)(src + p * G::kRow + 80);
                    const float v[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) u[k] = v[k];
                }
                epi_row<MODE, 8>(e, m0 + r, n, nv, t, u, sa, sb);
            }
        };
        stage_sums<0>(ep, acc, sh);
        half(0);
        if constexpr (MBLK == 4) {
            stage_sums<1>(ep, acc, sh);
            half(1);
        }
    }
    if (!epi_fwd(MODE) && e.sums) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int off = G::kLpr; off < 64; off <<= 1) {
                sa[k] += __shfl_xor(sa[k], off, 64);
                if (MODE == kEpiGluBwd) sb[k] += __shfl_xor(sb[k], off, 64);
            }
        if (r0 == 0 && nv > 0) {
            float* s = e.sums + srow * e.sum_cols + n;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < nv) {
                    s[k] = sa[k];
                    if (MODE == kEpiGluBwd) s[e.N + k] = sb[k];
                }
        }
    }
    return mag;
}

// ------------------------------------------------------------ 256-row tiles
// Grid, tiles and the narrower last round as gemm_nt_256, over the columns of B
// (kEpiGlu: of both matrices, in blocks of 16 in turn).
template <int MODE, int ACT, int TN>
__device__ __forceinline__ void ffn_tile(uint8_t* smem, int bid, int nb, const Epi& e, int tiles_m, int tiles_n, int col0) {
    constexpr bool kPair = MODE == kEpiGlu;
    const int w = threadIdx.x >> 6;
    const int g = __builtin_amdgcn_readfirstlane(w >> 2), sq = __builtin_amdgcn_readfirstlane(w & 3);
    int tm, tn;
    tile_of(bid, nb, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * kBM, n0 = col0 + tn * TN;
    const int wr0 = (sq >> 1) * 128 + g * 64, wc0 = (sq & 1) * (TN / 2);
    v4f acc[4][TN / 32];
    mm256_loop<epi_fa(MODE), FP8_E4M3, TN, kPair>(smem, e.A, e.B, (int)e.M, (int)e.N, (int)e.K, m0, n0, acc);
    // The main loop's last barrier follows every read of the operand tiles, so
    // group 0 stages its sums while group 1 issues its last MFMAs.
    static_assert(8 * 32 * (TN * 2 + 16) <= kSmemBytes - 64, "LDS budget");
    const int bq = e.q ? clamp_bias(*e.pred) : 0;
    const uint32_t mag = wave_epilogue<MODE, ACT, 4, TN / 32>(e, smem + w * 32 * (TN * 2 + 16), acc, m0 + wr0,
                                                              (n0 + wc0) / (kPair ? 2 : 1), 4 * tm + wr0 / 64, bq);
    if (e.q) {  // the workgroup's largest output for the exact bias
        uint32_t* wmx = (uint32_t*)(smem + kSmemBytes - 64);
        const uint32_t wv = wave_max_u32(mag);
        if ((threadIdx.x & 63) == 0) wmx[w] = wv;
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t b = 0;
#pragma unroll
            for (int v = 0; v < kMainThreads / 64; ++v) b = max(b, wmx[v]);
            e.parts[blockIdx.x] = b;
            if (blockIdx.x == 0) *e.used = bq;
        }
    }
}

// Workgroups below g1 take tiles 256 wide, the rest TN2 wide (see mm256_split).
template <int MODE, int ACT, int TN2>
__global__ __launch_bounds__(kMainThreads) void ffn_256(Epi e, int tiles_m, int tiles_n, int g1, int tiles_n2) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kSmemBytes];
    const int b = blockIdx.x;
    if (b < g1) ffn_tile<MODE, ACT, 256>(smem, b, g1, e, tiles_m, tiles_n, 0);
    else ffn_tile<MODE, ACT, TN2>(smem, b - g1, (int)gridDim.x - g1, e, tiles_m, tiles_n2, tiles_n * kBN);
}

// ------------------------------------------------------------ any K
template <int MODE, int BM, int BN, int WT>
__global__ __launch_bounds__((BM / WT) * (BN / WT) * 64) void ffn_ragged(Epi e, int tiles_m, int tiles_n) {
    constexpr bool kPair = MODE == kEpiGlu;
    constexpr int kWaves = (BM / WT) * (BN / WT), kStage = (BM + BN) * kRk, kEpWave = 32 * (WT * 4 + 16);
    constexpr int kSmem = 2 * kStage > kWaves * kEpWave ? 2 * kStage : kWaves * kEpWave;
    __shared__ __attribute__((aligned(128))) uint8_t smem[kSmem];
    const int w = threadIdx.x >> 6;
    int tm, tn;
    tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int wr0 = (w / (BN / WT)) * WT, wc0 = (w % (BN / WT)) * WT;
    v4f acc[WT / 16][WT / 16];
    ragged_loop<epi_fa(MODE), FP8_E4M3, BM, BN, WT, kPair>(smem, e.A, e.B, e.M, e.N, e.K, m0, n0, acc);
    wave_epilogue<MODE, -1, WT / 16, WT / 16>(e, smem + w * kEpWave, acc, m0 + wr0, (n0 + wc0) / (kPair ? 2 : 1),
                                              (m0 + wr0) / WT, 0);
}

// ------------------------------------------------------------ launches
template <int MODE>
void launch_ragged(const Epi& e, hipStream_t s) {
    const int64_t cols = epi_b_cols(MODE, e.N);
    if (epi_big_tiles(e.M, cols)) {
        const int tm = (int)((e.M + 255) / 256), tn = (int)((cols + 127) / 128);
        hipLaunchKernelGGL((ffn_ragged<MODE, 256, 128, 64>), dim3((unsigned)((int64_t)tm * tn)), dim3(512), 0, s, e, tm, tn);
    } else {
        const int tm = (int)((e.M + 63) / 64), tn = (int)((cols + 63) / 64);
        hipLaunchKernelGGL((ffn_ragged<MODE, 64, 64, 32>), dim3((unsigned)((int64_t)tm * tn)), dim3(256), 0, s, e, tm, tn);
    }
}

template <int MODE, int ACT>
void launch_256(const Epi& e, hipStream_t s) {
    const int64_t cols = epi_b_cols(MODE, e.N);
    const int tiles_m = (int)((e.M + kBM - 1) / kBM), tiles_n = (int)((cols + kBN - 1) / kBN);
    int ndp, tw, tn2;
    mm256_split(tiles_m, tiles_n, cols, ndp, tw, tn2);
    const int g1 = tiles_m * ndp;
    const dim3 grid(g1 + tiles_m * tn2), block(kMainThreads);
    if (tw == 64) hipLaunchKernelGGL((ffn_256<MODE, ACT, 64>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);
    else if (tw == 128) hipLaunchKernelGGL((ffn_256<MODE, ACT, 128>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);
    else hipLaunchKernelGGL((ffn_256<MODE, ACT, 192>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);  // tw == 0: none of these
}

template <int MODE>
void launch_mode(bool ragged, const Epi& e, hipStream_t s) {
    if (ragged) return launch_ragged<MODE>(e, s);
    switch (e.act) {
        case FP8_ACT_RELU: launch_256<MODE, FP8_ACT_RELU>(e, s); break;
        case FP8_ACT_GELU: launch_256<MODE, FP8_ACT_GELU>(e, s); break;
        case FP8_ACT_GELU_TANH: launch_256<MODE, FP8_ACT_GELU_TANH>(e, s); break;
        case FP8_ACT_SILU: launch_256<MODE, FP8_ACT_SILU>(e, s); break;
        default: launch_256<MODE, FP8_ACT_NONE>(e, s);
    }
}

}  // namespace
}  // namespace fp8lin
