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
// The sums go through LDS, 16 rows of a wave at a time, so that a lane gets eight
// consecutive columns of a row: every global access is then a 16-byte piece of a
// row run.
//
// What bounds it: the matrix cores, and after them the epilogue, which a workgroup has
// to itself (its operand stages take the whole LDS, so no second one is there to
// multiply meanwhile).  What an output of 4096 x 16384 takes besides its products (the
// time at K = 4096 and 8192 carried on to K = 0, in us; in brackets its bytes at the
// rate of a device copy):
//   plain matmul 41 (27); bias, GELU 65 (27); the same keeping z 82 (54), with codes
//   both ways 110 (81); gated pair 38 (13), keeping both 48 (40), with codes 65 (54);
//   backward GELU 89 (54), with the bias gradient 94, with codes 129 (81); gated
//   backward 151 (108), with codes 234 (162).
// 4096 x 13824 x 5120 with GELU, z and codes: 278 us of which 195 are its products at
// the best rate of the plain matmul; 4096 x 28672 x 8192 gated: 1396 (1293).
#pragma once

#include "fp8lin_epilogue.h"
#include "fp8lin_glue.h"
#include "fp8lin_mm_256.h"
#include "fp8lin_mm_ragged.h"

namespace fp8lin {
namespace {

constexpr int pow2_up(int n) { return n <= 1 ? 1 : 2 * pow2_up((n + 1) / 2); }

// Geometry of a wave's epilogue: MBLK x NBLK blocks of 16 x 16 sums, staged 16 rows
// at a time; an eight of columns to a lane, kNp consecutive rows of it one after
// another (so that their codes' bytes end in one lane for the transposed copy).
template <int MODE, int NBLK>
struct EpiGeo {
    static constexpr bool kPair = MODE == kEpiGlu;
    static constexpr int kRow = NBLK <= 2 ? 128 : NBLK <= 4 ? 256 : 512;  // staging row, bytes
    static constexpr int kOct = kPair ? NBLK : 2 * NBLK;  // eights of columns in a row
    static constexpr int kLpr = kOct <= 4 ? 4 : pow2_up(kOct), kNp = kLpr / 4;  // lanes a row, rows of a lane
    static_assert((!kPair || NBLK % 2 == 0) && kLpr <= 16, "blocks of a wave");
};

// 16-byte chunk c of staging row r (r < 16) is stored at chunk c ^ stage_swz(r): a
// write has lanes on 16 rows and two neighbouring chunks, a read lanes on two rows
// four apart and every second chunk, and either way the 16 lanes of a phase (see
// fp8lin_gemm.hip) hit 16 distinct groups of banks.
template <int ROW>
__device__ __forceinline__ int stage_swz(int r) {
    return (((r >> 2) & 1) | ((r & 3) << 1) | (((r >> 2) ^ (r >> 3)) & 1) << 3) & (ROW / 16 - 1);
}

// Stages rows 16 i .. 16 i + 15 of a wave's sums, unscaled by 2^sh, for its other lanes
// to read, after they have read the sixteen before.
template <int ROW, int NBLK>
__device__ __forceinline__ void stage_sums(uint8_t* ep, const v4f (&acc)[NBLK], int sh, int lane) {
    const int frow = lane & 15, fg = lane >> 4, z = stage_swz<ROW>(frow);
    wave_lds_order();
#pragma unroll
    for (int j = 0; j < NBLK; ++j) {
        const v4f a = acc[j];
        *(float4*)(ep + frow * ROW + (((4 * j + fg) ^ z) << 4)) =
            make_float4(ldexpf(a[0], sh), ldexpf(a[1], sh), ldexpf(a[2], sh), ldexpf(a[3], sh));
    }
    wave_lds_order();
}

// Eight staged sums of row r from chunk c on.
template <int ROW>
__device__ __forceinline__ void staged8(const uint8_t* ep, int r, int c, float4& a, float4& b) {
    const int z = stage_swz<ROW>(r);
    a = *(const float4*)(ep + r * ROW + ((c ^ z) << 4));
    b = *(const float4*)(ep + r * ROW + (((c + 1) ^ z) << 4));
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

// Transposed codes of a tile in LDS (stored from the registers, 8 bytes of each column 32
// KB apart, they took 70 to 170 us more at 4096 rows): a column of codes is 256 bytes, one a row of the
// tile, its 16-byte chunk q stored at chunk q ^ code_swz(column): the lanes of a
// write (columns eight apart) and of a read (one column) hit distinct banks.
__device__ __forceinline__ int code_swz(int col) { return (col ^ (col >> 3)) & 15; }

// The codes c of NP consecutive tile rows from `row` on of eight columns from `col` on.
template <int NP>
__device__ __forceinline__ void put_codes(uint8_t* cs, int row, int col, const uint2 (&c)[NP]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = i < NP ? (h ? c[i % NP].y : c[i % NP].x) : 0u;
        transpose4(t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = col + 4 * h + i;
            uint8_t* p = cs + n * 256 + (((row >> 4) ^ code_swz(n)) << 4) + (row & 15);
            if (NP == 4) *(uint32_t*)p = t[i];
            else if (NP == 2) *(uint16_t*)p = (uint16_t)t[i];
            else *p = (uint8_t)t[i];
        }
    }
}

// Columns 0 .. cols - 1 of those codes to the transposed copy at q (the tile's first
// column and row), rows of them in the matrix.
__device__ __forceinline__ void store_codes(const uint8_t* cs, uint8_t* q, int64_t ld, int cols, int rows, int tid) {
    const int c16 = tid & 15;
    for (int n = tid >> 4; n < cols; n += kMainThreads / 16) {
        const uint4 v = *(const uint4*)(cs + n * 256 + ((c16 ^ code_swz(n)) << 4));
        uint8_t* p = q + n * ld + c16 * 16;
        const int k = rows - c16 * 16;
        if (k >= 16) {
            st_stream(p, v);
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < k) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
        }
    }
}

// What a wave's epilogue needs beside the sums.
template <int MODE, int NBLK>
struct EpiWave {
    static constexpr int kNp = EpiGeo<MODE, NBLK>::kNp;
    int lane;
    uint8_t *ep, *cs;        // 16 staging rows of its own; the tile's transposed codes
    int64_t m0, n0;          // its first row and column of the output (uniform)
    int rows;                // its rows in the matrix
    int row0, col0;          // its first row and column of the tile's output
    bool active;             // this lane's eight columns are in the matrix
    int sh, bq;
    float ba[8], bu[8];      // bias
    float sa[8], sb[8];      // column sums
    uint32_t mag;            // largest output (bf16 pattern)
};

// What the p-th of a lane's rows among rows 16 i .. 16 i + 15 needs from memory (bf16).
template <int MODE, int NBLK>
__device__ __forceinline__ void epi_load(const Epi& e, const EpiWave<MODE, NBLK>& w, int i, int p, uint4& x, uint4& u) {
    using G = EpiGeo<MODE, NBLK>;
    if (epi_fwd(MODE) && !(MODE == kEpiAct && e.res)) return;
    const int oct = w.lane & (G::kLpr - 1), r0 = w.lane / G::kLpr * G::kNp;
    const uint32_t ld = (uint32_t)(MODE == kEpiAct ? e.ldres : e.ldz);
    const uint16_t* src = (MODE == kEpiAct ? (const uint16_t*)e.res : e.z) + w.m0 * ld + w.n0;
    const uint32_t at = (uint32_t)min(16 * i + r0 + p, w.rows - 1) * ld + 8 * oct;
    x = ld_stream(src + at);
    if (MODE == kEpiGluBwd) u = ld_stream(src + e.N + at);
}

// Rows 16 i .. 16 i + 15 of a wave, where every lane's eight columns are all in
// the matrix or all outside and the output is bf16.  The lanes' offsets from the wave's
// first element of a tensor are 32-bit.  pre, pre2: epi_load of each row; those of the
// rows AHEAD sixteens on take their place as they are used (LEFT sixteens are left).
template <int MODE, int ACT, int AHEAD, int LEFT, int NBLK>
__device__ __forceinline__ void epi_rows(const Epi& e, EpiWave<MODE, NBLK>& w, const v4f (&acc)[NBLK], int i,
                                         uint4 (&pre)[EpiGeo<MODE, NBLK>::kNp],
                                         uint4 (&pre2)[EpiGeo<MODE, NBLK>::kNp]) {
    using G = EpiGeo<MODE, NBLK>;
    constexpr bool kPair = G::kPair, kTwo = MODE == kEpiGluBwd;
    constexpr int kNp = G::kNp, kFmt = epi_fwd(MODE) ? FP8_E4M3 : FP8_E5M2;
    const int oct = w.lane & (G::kLpr - 1), r0 = w.lane / G::kLpr * kNp;
    const uint32_t col = 8 * oct;
    stage_sums<G::kRow>(w.ep, acc, w.sh, w.lane);
    if (!w.active) return;
    const int chunk = kPair ? (oct >> 1) * 8 + (oct & 1) * 2 : oct * 2;  // of the first sums; a pair's others 4 on
    const bool res = MODE == kEpiAct && e.res;
    uint16_t* ob = (uint16_t*)e.out + w.m0 * e.ldo + w.n0;
    uint16_t* kb = e.keep + w.m0 * e.ldkeep + w.n0;
    uint8_t* qb = e.q + w.m0 * e.ldq + w.n0;
    uint2 c8[kNp];
    float4 st[kPair ? 4 : 2];  // a row's sums, read while the row before is computed
    auto fetch = [&](int p) {
        staged8<G::kRow>(w.ep, r0 + p, chunk, st[0], st[1]);
        if (kPair) staged8<G::kRow>(w.ep, r0 + p, chunk + 4, st[kPair ? 2 : 0], st[kPair ? 3 : 1]);
    };
    fetch(0);
#pragma unroll
    for (int p = 0; p < kNp; ++p) {
        float t[8] = {st[0].x, st[0].y, st[0].z, st[0].w, st[1].x, st[1].y, st[1].z, st[1].w}, u[8], x[8], y[8], f, d;
        if (kPair) {
            const float4 u0 = st[kPair ? 2 : 0], u1 = st[kPair ? 3 : 1];
            const float v[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = v[k];
        }
        if (p + 1 < kNp) fetch(p + 1);
        if (!epi_fwd(MODE) || res) unpack8(pre[p], x);
        if (kTwo) unpack8(pre2[p], u);
        if (AHEAD < LEFT) epi_load(e, w, i + AHEAD, p, pre[p], pre2[p]);
        const int r = 16 * i + r0 + p;
        const bool in = r < w.rows;
        uint4 o, o2 = make_uint4(0u, 0u, 0u, 0u);
        if (epi_fwd(MODE)) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                t[k] += w.ba[k];
                if (kPair) u[k] += w.bu[k];
            }
            if (e.keep) {
                o = pack8(t);
                if (kPair) o2 = pack8(u);
                if (in) {
                    st_stream(kb + ((uint32_t)r * (uint32_t)e.ldkeep + col), o);
                    if (kPair) st_stream(kb + e.N + ((uint32_t)r * (uint32_t)e.ldkeep + col), o2);
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                act_t<ACT>(t[k], &f, &d);
                y[k] = kPair ? f * u[k] : res ? f + x[k] : f;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                act_t<ACT>(x[k], &f, &d);
                if (kTwo) x[k] = t[k] * f;
                y[k] = (kTwo ? t[k] * u[k] : t[k]) * d;
            }
            if (e.sums && in) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    w.sa[k] += y[k];
                    if (kTwo) w.sb[k] += x[k];
                }
            }
            if (kTwo) o2 = pack8(x);
        }
        o = pack8(y);
        if (in) {
            st_stream(ob + ((uint32_t)r * (uint32_t)e.ldo + col), o);
            if (kTwo) st_stream(ob + e.N + ((uint32_t)r * (uint32_t)e.ldo + col), o2);
        }
        if (e.q) {
            c8[p] = codes8<kFmt>(o, w.bq);
            if (in) w.mag = max(w.mag, mag8(o));
            if (in) st8_any(qb + ((uint32_t)r * (uint32_t)e.ldq + col), c8[p].x, c8[p].y);
            if (kTwo) {
                const uint2 c = codes8<kFmt>(o2, w.bq);
                if (in) w.mag = max(w.mag, mag8(o2));
                if (in) st8_any(qb + e.N + ((uint32_t)r * (uint32_t)e.ldq + col), c.x, c.y);
            }
        }
    }
    if (!kTwo && e.qT) put_codes<kNp>(w.cs, w.row0 + 16 * i + r0, w.col0 + 8 * oct, c8);
}

// The epilogue of one wave: MBLK x NBLK blocks of 16 x 16 sums (laid out as in
// mm256_loop) of rows m0 .., columns n0 .. of the output (with kEpiGlu NBLK / 2
// blocks of columns of each projection); srow: its row of the column sums.  ACT < 0:
// the activation is e.act, and the epilogue exists once, in a loop (tiles cut by the
// matrix's last columns, any K).  What is read from memory is under way while the
// sixteen rows before are computed.  4096 x 13824 x 5120, GELU and z: 256 us; fp32 output
// 266, 13821 columns 270, K = 5000 374.
template <int MODE, int ACT, int MBLK, int NBLK>
__device__ __forceinline__ void wave_epilogue(const Epi& e, EpiWave<MODE, NBLK>& w, const v4f (&acc)[MBLK][NBLK], int64_t srow) {
    using G = EpiGeo<MODE, NBLK>;
    constexpr int kNp = G::kNp;
    static_assert(MBLK <= 4, "rows of a wave");
    const int oct = w.lane & (G::kLpr - 1), r0 = w.lane / G::kLpr * kNp;
    const int64_t n = w.n0 + 8 * oct;
    const int nv = oct < G::kOct ? (int)min((int64_t)8, e.N - n) : 0;
    w.sh = -(*e.ba + *e.bb);
    w.rows = (int)min((int64_t)(16 * MBLK), e.M - w.m0);
    w.mag = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) w.ba[k] = w.bu[k] = w.sa[k] = w.sb[k] = 0.0f;
    if (ACT >= 0 && e.fast && !__any(nv > 0 && nv < 8)) {
        constexpr int kA = ACT >= 0 ? ACT : 0;
        w.active = nv > 0;
        if (epi_fwd(MODE) && e.bias && w.active) {
            ld_vals<8>(e.bias, n, e.bias_dt, 8, w.ba);
            if (MODE == kEpiGlu) ld_vals<8>(e.bias, e.N + n, e.bias_dt, 8, w.bu);
        }
        if (w.rows > 0) {
            // of a gated block's backward pass, with two tensors to read, sixteen rows ahead;
            // otherwise 32 (the registers that the sums leave: with 32 there, too, up to 128
            // are spilled and 4096 x 11008 x 4096 takes 270 us instead of 262)
            constexpr int kAhead = MODE == kEpiGluBwd ? 1 : 2;
            uint4 x[kAhead][kNp], u[kAhead][kNp];
            if (w.active) {
#pragma unroll
                for (int i = 0; i < kAhead && i < MBLK; ++i)
#pragma unroll
                    for (int p = 0; p < kNp; ++p) epi_load(e, w, i, p, x[i][p], u[i][p]);
            }
            __builtin_amdgcn_sched_barrier(0);
            epi_rows<MODE, kA, kAhead, MBLK>(e, w, acc[0], 0, x[0], u[0]);
            if constexpr (MBLK > 1) epi_rows<MODE, kA, kAhead, MBLK - 1>(e, w, acc[1], 1, x[1 % kAhead], u[1 % kAhead]);
            if constexpr (MBLK > 2) epi_rows<MODE, kA, kAhead, MBLK - 2>(e, w, acc[2], 2, x[0], u[0]);
            if constexpr (MBLK > 3) epi_rows<MODE, kA, kAhead, MBLK - 3>(e, w, acc[3], 3, x[1 % kAhead], u[1 % kAhead]);
        }
    } else {
        const int chunk = G::kPair ? (oct >> 1) * 8 + (oct & 1) * 2 : oct * 2;
#pragma unroll
        for (int i = 0; i < MBLK; ++i) {
            stage_sums<G::kRow>(w.ep, acc[i], w.sh, w.lane);
            const int r = 16 * i + r0;
#pragma unroll 1
            for (int p = 0; p < kNp; ++p) {
                if (nv <= 0 || r + p >= w.rows) continue;
                float4 t0, t1, u0, u1;
                staged8<G::kRow>(w.ep, r0 + p, chunk, t0, t1);
                float t[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w}, u[8];
                if (G::kPair) {
                    staged8<G::kRow>(w.ep, r0 + p, chunk + 4, u0, u1);
                    const float v[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) u[k] = v[k];
                }
                float y[8], x[8];
                epi_row<MODE, 8>(e, w.m0 + r + p, n, nv, t, u, w.sa, w.sb, y, x);
            }
        }
    }
    if (!epi_fwd(MODE) && e.sums) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int off = G::kLpr; off < 64; off <<= 1) {
                w.sa[k] += __shfl_xor(w.sa[k], off, 64);
                if (MODE == kEpiGluBwd) w.sb[k] += __shfl_xor(w.sb[k], off, 64);
            }
        if (r0 == 0 && nv > 0) {
            float* s = e.sums + srow * e.sum_cols + n;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < nv) {
                    s[k] = w.sa[k];
                    if (MODE == kEpiGluBwd) s[e.N + k] = w.sb[k];
                }
        }
    }
}

// ------------------------------------------------------------ 256-row tiles
// The kernel's first argument, read from its segment where this is called.
__device__ __forceinline__ Epi late_args() {
    struct Words {
        uint64_t w[sizeof(Epi) / 8];
    } v;
    static_assert(sizeof(Epi) % 8 == 0, "argument words");
    auto p = (const __attribute__((address_space(4))) uint64_t*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("; arguments of the epilogue" : "+s"(p));
#pragma unroll
    for (size_t i = 0; i < sizeof(Epi) / 8; ++i) v.w[i] = p[i];
    return __builtin_bit_cast(Epi, v);
}

// The thread's number, likewise: what the epilogue derives from it is not kept from
// the start.
__device__ __forceinline__ int late_thread() {
    int t = threadIdx.x;
    asm volatile("; thread of the epilogue" : "+v"(t));
    return t;
}

// Grid, tiles and the narrower last round as gemm_nt_256, over the columns of B
// (kEpiGlu: of both matrices, in blocks of 16 in turn).
template <int MODE, int ACT, int TN>
__device__ __forceinline__ void ffn_tile(uint8_t* smem, int bid, int nb, const Epi& args, int tiles_m, int tiles_n, int col0) {
    constexpr bool kPair = MODE == kEpiGlu;
    const int w = threadIdx.x >> 6;
    const int g = __builtin_amdgcn_readfirstlane(w >> 2), sq = __builtin_amdgcn_readfirstlane(w & 3);
    int tm, tn;
    tile_of(bid, nb, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * kBM, n0 = col0 + tn * TN;
    const int wr0 = (sq >> 1) * 128 + g * 64, wc0 = (sq & 1) * (TN / 2);
    v4f acc[4][TN / 32];
    mm256_loop<epi_fa(MODE), FP8_E4M3, TN, kPair>(smem, args.A, args.B, (int)args.M, (int)args.N, (int)args.K, m0, n0, acc);
    // The epilogue's arguments are read here: held in registers through the main loop
    // they would be spilled there (a spill costs it its place in the schedule: the plain
    // matmul of 4096 x 28672 x 8192 went from 608 to 580 us without any).  What is left:
    // with kEpiAct in tiles 128 and 192 wide 4 to 9 scalar registers, with 128 also 20 bytes
    // of scratch a lane.
    const Epi e = late_args();
    const int tid = late_thread(), lane = tid & 63;
    // The main loop's last barrier follows every read of the operand tiles, so
    // group 0 stages its sums while group 1 issues its last MFMAs.
    // LDS: the waves' staging rows, the transposed codes, the waves' maxima.
    constexpr int kEpWave = 16 * EpiGeo<MODE, TN / 32>::kRow, kCols = kPair ? TN / 2 : TN;
    static_assert(8 * kEpWave + kCols * 256 + 64 <= kSmemBytes && 8 * kEpWave % 16 == 0, "LDS budget");
    EpiWave<MODE, TN / 32> wv;
    wv.lane = lane;
    wv.ep = smem + w * kEpWave;
    wv.cs = smem + 8 * kEpWave;
    wv.row0 = wr0;
    wv.col0 = wc0 / (kPair ? 2 : 1);
    wv.m0 = m0 + wr0;
    wv.n0 = n0 / (kPair ? 2 : 1) + wv.col0;
    wv.bq = e.q ? clamp_bias(*e.pred) : 0;
    wave_epilogue<MODE, ACT>(e, wv, acc, 4 * tm + wr0 / 64);
    if (e.q) {
        // the transposed codes of whole columns, and the workgroup's largest output
        // for the exact bias
        uint32_t* wmx = (uint32_t*)(smem + kSmemBytes - 64);
        const uint32_t mx = wave_max_u32(wv.mag);
        if (lane == 0) wmx[w] = mx;
        __syncthreads();
        const int64_t nt = n0 / (kPair ? 2 : 1);
        const int cols = (int)min((int64_t)kCols, e.N - nt), rows = min(kBM, (int)e.M - m0);
        if (MODE != kEpiGluBwd && e.qT) store_codes(wv.cs, e.qT + nt * e.ldqT + m0, e.ldqT, cols, rows, tid);
        if (tid == 0) {
            uint32_t b = 0;
#pragma unroll
            for (int v = 0; v < kMainThreads / 64; ++v) b = max(b, wmx[v]);
            e.parts[blockIdx.x] = b;
            if (blockIdx.x == 0) *e.used = wv.bq;
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
    constexpr int kWaves = (BM / WT) * (BN / WT), kStage = (BM + BN) * kRk, kEpWave = 16 * EpiGeo<MODE, WT / 16>::kRow;
    constexpr int kSmem = 2 * kStage > kWaves * kEpWave ? 2 * kStage : kWaves * kEpWave;
    __shared__ __attribute__((aligned(128))) uint8_t smem[kSmem];
    const int w = threadIdx.x >> 6;
    int tm, tn;
    tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int wr0 = (w / (BN / WT)) * WT, wc0 = (w % (BN / WT)) * WT;
    v4f acc[WT / 16][WT / 16];
    ragged_loop<epi_fa(MODE), FP8_E4M3, BM, BN, WT, kPair>(smem, e.A, e.B, e.M, e.N, e.K, m0, n0, acc);
    EpiWave<MODE, WT / 16> wv;
    wv.lane = threadIdx.x & 63;
    wv.ep = smem + w * kEpWave;
    wv.m0 = m0 + wr0;
    wv.n0 = (n0 + wc0) / (kPair ? 2 : 1);
    wave_epilogue<MODE, -1>(e, wv, acc, (m0 + wr0) / WT);
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
