// The small-tile matmul kernel (described in fp8lin_gemm_stream.hip), with the plain
// epilogue or another.  Internal, not part of the ABI.
#pragma once

#include "fp8lin_mm.h"

namespace fp8lin {
namespace {

constexpr int kSlBuf = 3;

// Waves 0-3 multiply; with more than 16 rows of A waves 4-7 copy, otherwise
// the multiplying waves copy too (see the main loop).
constexpr bool copy_waves(int mb) { return mb > 1; }
constexpr int stream_threads(int mb) { return copy_waves(mb) ? 512 : 256; }
constexpr int stream_kc(int mb, int nb) { return mb + nb <= 6 ? 512 : mb + nb <= 12 ? 256 : 128; }

// Tile shapes (16-row blocks of A and of B) the kernel is built for: those the
// rule below chooses somewhere for 1 to 2048 rows and weights of 128 to 57344
// ((1, 4), (4, 2) and (8, 4) only for calls that take the amax).
#define FP8LIN_STREAM_TILES(X)                                                                             \
    X(1, 1) X(1, 2) X(1, 3) X(1, 4) X(1, 5) X(1, 6) X(1, 8) X(2, 1) X(2, 2) X(2, 3) X(2, 4) X(2, 6) X(2, 8)  \
    X(3, 1) X(3, 2) X(3, 3) X(3, 4) X(3, 6) X(3, 8) X(4, 2) X(4, 4) X(4, 6) X(4, 8) X(5, 2) X(5, 4) X(5, 6) \
    X(6, 4) X(6, 6) X(8, 4) X(8, 8) X(10, 6)

// One tile of 16 MB x 16 NB outputs.  E: what becomes of the sums.  E::kPlain: as
// MmArgs says (gemm_nt_stream's own epilogue); otherwise E::finish gets them in LDS, as
// [slot][16-row block][16-column block][lane] partial sums over k, which it adds
// over the slots.  E::kPair: B is two matrices of N rows each, one after the other,
// and a tile takes blocks of 16 rows from them in turn, from row n0 / 2 on (NB even).
template <int FA, int FB, int MB, int NB, class E>
__global__ __launch_bounds__(stream_threads(MB)) void gemm_nt_stream(typename E::Args p, int tiles_m, int tiles_n, int nt) {
    constexpr bool kPair = E::kPair;
    constexpr int kRowsB = 16 * NB, kRows = 16 * (MB + NB);
    constexpr int kKC = stream_kc(MB, NB);
    constexpr int kStage = kRows * kKC, kCpr = kKC / 16, kRpi = 64 / kCpr;  // chunks per row, rows per copy
    constexpr int kNiw = kRows / kRpi / 4;                                  // copies per wave and stage
    constexpr int kSlots = kKC / 128;
    constexpr int kWn = kSlots == 4 ? 1 : 2, kWm = kSlots == 1 ? 2 : 1;  // waves over the tile's columns, rows
    constexpr int kNbw = NB / kWn, kMbw = MB / kWm;
    static_assert(kRows % (4 * kRpi) == 0 && NB % kWn == 0 && MB % kWm == 0, "tile split");
    static_assert(kSlBuf * kStage <= 160 * 1024 && (kSlots == 1 || kSlots * MB * NB * 1024 <= kSlBuf * kStage), "LDS budget");
    __shared__ __attribute__((aligned(1024))) uint8_t sm[kSlBuf * kStage];
    __shared__ uint32_t wmx[8];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int M = (int)p.M, N = (int)p.N, K = (int)p.K;
    // consecutive tiles of one XCD share their B rows
    const int x = blockIdx.x & 7, per = gridDim.x >> 3, rem = gridDim.x & 7;
    const int tile = x * per + min(x, rem) + (blockIdx.x >> 3);
    int tm = tile % tiles_m, tn = tile / tiles_m;
    if (kSlots == 1) tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * (16 * MB), n0 = tn * kRowsB;
    // 16-byte chunk c of LDS row r is stored at chunk c ^ swz(r)
    auto swz = [](int r) { return kKC == 128 ? chunk_swz(r) : r & 15; };

    // copy t of this wave: LDS rows kRpi d .. (d = kNiw w + t), B rows first;
    // rows past the matrix edge read the last row (their outputs are not stored)
    const int lrow = lane / kCpr, lchunk = lane % kCpr;
    uint32_t voff[kNiw];
#pragma unroll
    for (int t = 0; t < kNiw; ++t) {
        const int r = ((w & 3) * kNiw + t) * kRpi + lrow;
        const int src = r >= kRowsB ? min(m0 + r - kRowsB, M - 1) - m0
                        : kPair     ? min(n0 / 2 + pair_row(r), N - 1) - n0 / 2
                                    : min(n0 + r, N - 1) - n0;
        voff[t] = (uint32_t)(src * K + ((lchunk ^ swz(r)) << 4));
    }
    const uint8_t* baseA = p.A + (int64_t)m0 * K;
    const uint8_t* baseB = p.B + (int64_t)(kPair ? n0 / 2 : n0) * K;
    const uint32_t lds0 = lds_addr(sm);
    const int nst = (K + kKC - 1) / kKC;
    auto issue = [&](int st) {
        const int buf = st % kSlBuf, end = K - st * kKC - 16;  // offset of the row's last chunk
        const bool part = end + 16 < kKC;
#pragma unroll
        for (int t = 0; t < kNiw; ++t) {
            const int d = (w & 3) * kNiw + t;
            const uint32_t dst = __builtin_amdgcn_readfirstlane(lds0 + buf * kStage + d * 1024);
            uint32_t v = voff[t];
            if (part) {  // chunks past the row end re-read its last one (never multiplied)
                const int c = (lchunk ^ swz(d * kRpi + lrow)) << 4;
                v -= (uint32_t)max(0, c - end);
            }
            // a copy's rows lie in one block of 16: which of the pair is wave-uniform
            const uint8_t* b = baseB + (kPair && ((d * kRpi >> 4) & 1) ? (int64_t)N * K : 0);
            if (d * kRpi >= kRowsB) lds_dma16_s(baseA + (int64_t)st * kKC, v, dst);
            else if (nt) lds_dma16_nt(b + (int64_t)st * kKC, v, dst);
            else lds_dma16_s(b + (int64_t)st * kKC, v, dst);
        }
    };

    const int frow = lane & 15, fg = lane >> 4;
    const int slot = w % kSlots, part = (w & 3) / kSlots;
    const int nb0 = part % kWn * kNbw, mb0 = part / kWn * kMbw;  // this wave's blocks of the tile
    const int fo0 = frow * kKC + (((slot * 8 + 2 * fg) ^ swz(frow)) << 4);
    const int fo1 = frow * kKC + (((slot * 8 + 2 * fg + 1) ^ swz(frow)) << 4);
    v4f acc[kMbw][kNbw];
#pragma unroll
    for (int i = 0; i < kMbw; ++i)
#pragma unroll
        for (int j = 0; j < kNbw; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](int st) {
        if (st * kKC + slot * 128 >= K) return;
        const uint8_t* sb = sm + (st % kSlBuf) * kStage + nb0 * 16 * kKC;
        const uint8_t* sa = sm + (st % kSlBuf) * kStage + (kRowsB + mb0 * 16) * kKC;
        v8i bf[kNbw];
#pragma unroll
        for (int j = 0; j < kNbw; ++j) bf[j] = ld_frag(sb + j * 16 * kKC, fo0, fo1);
#pragma unroll
        for (int i = 0; i < kMbw; ++i) {
            const v8i af = ld_frag(sa + i * 16 * kKC, fo0, fo1);
#pragma unroll
            for (int j = 0; j < kNbw; ++j) acc[i][j] = mfma16<FB, FA>(bf[j], af, acc[i][j]);
        }
        wait_lgkmcnt0();  // the next barrier frees this buffer
    };
    // wait until stage st has landed, stages up to `issued` being on their way
    auto landed = [&](int st, int issued) {
        if (st < issued) wait_vmcnt<kNiw>();
        else wait_vmcnt<0>();
    };
    if (copy_waves(MB)) {
        // Between barriers st and st + 1 the multiplying waves take stage st
        // and the copying waves issue stage st + 2 into the buffer of stage
        // st - 1 and wait for stage st + 1: an issue that stalls for room
        // among the outstanding fills stalls no multiplication (100 x 12288 x
        // 4096: 23.6 -> 18.0 us, 512 x 8192 x 8192: 93 -> 61 us).
        if (w >= 4) {
            if (nst > 0) issue(0);
            if (nst > 1) issue(1);
            landed(0, nst - 1);
            ws_barrier();
            for (int st = 0; st < nst; ++st) {
                if (st + 2 < nst) issue(st + 2);
                landed(st + 1, nst - 1);
                ws_barrier();
            }
        } else {
            ws_barrier();
            for (int st = 0; st < nst; ++st) {
                multiply(st);
                ws_barrier();
            }
        }
    } else {
        // Few MFMAs per stage: copying waves of their own gain nothing and
        // cost 1-5 % of a stream from HBM (16 x 57344 x 8192: 74.8 against
        // 79.1 us).
        if (nst > 0) issue(0);
        if (nst > 1) issue(1);
        for (int st = 0; st < nst; ++st) {
            landed(st, nst - 1);
            ws_barrier();
            // the buffer of stage st - 1, which every wave has finished reading
            if (st + 2 < nst) issue(st + 2);
            multiply(st);
        }
        ws_barrier();
    }
    if constexpr (!E::kPlain) {
        // each block's partial sums to the wave that takes it
        v4f* red = (v4f*)sm;  // [slot][16-row block][16-column block][lane]
        static_assert(kSlots * MB * NB * 1024 <= kSlBuf * kStage && (!kPair || NB % 2 == 0), "LDS budget");
        if (w < 4) {
#pragma unroll
            for (int i = 0; i < kMbw; ++i)
#pragma unroll
                for (int j = 0; j < kNbw; ++j) red[((slot * MB + mb0 + i) * NB + nb0 + j) * 64 + lane] = acc[i][j];
        }
        __syncthreads();
        E::template finish<MB, NB, kSlots>(p, red, wmx, m0, n0);
    } else {
        uint32_t mx = 0;
        const int bb = *p.bb;
        auto put = [&](int mb, int nb, v4f sum) {
            const int64_t m = m0 + mb * 16 + frow, n = n0 + nb * 16 + fg * 4;
            if (n >= N) return;
            const int sh = row_shift(p.ba, p.ba_rows, bb, m, M);
            mx = max(mx, p.out_dt == FP8_DT_BF16 ? store4<FP8_DT_BF16>(p.C, N, m, n, M, N, sum, sh)
                                                 : store4<FP8_DT_F32>(p.C, N, m, n, M, N, sum, sh));
        };
        if (kSlots == 1) {
            if (w < 4) {
#pragma unroll
                for (int i = 0; i < kMbw; ++i)
#pragma unroll
                    for (int j = 0; j < kNbw; ++j) put(mb0 + i, nb0 + j, acc[i][j]);
            }
        } else {
            v4f* red = (v4f*)sm;  // [slot][16-row block][16-column block][lane]
            if (w < 4) {
#pragma unroll
                for (int i = 0; i < kMbw; ++i)
#pragma unroll
                    for (int j = 0; j < kNbw; ++j) red[((slot * MB + i) * NB + nb0 + j) * 64 + lane] = acc[i][j];
            }
            __syncthreads();
            for (int b = w; b < MB * NB; b += stream_threads(MB) / 64) {
                v4f sum = red[b * 64 + lane];
#pragma unroll
                for (int s = 1; s < kSlots; ++s) sum += red[(s * MB * NB + b) * 64 + lane];
                put(b / NB, b % NB, sum);
            }
        }
        if (p.with_amax) {
            const uint32_t wv = wave_max_u32(mx);
            if (lane == 0) wmx[w] = wv;
            __syncthreads();
            if (threadIdx.x == 0) {
                uint32_t b = 0;
#pragma unroll
                for (int v = 0; v < stream_threads(MB) / 64; ++v) b = max(b, wmx[v]);
                fold_amax(canon_amax(b), p.amax, p.bo);
            }
        }
    }
}

}  // namespace
}  // namespace fp8lin
