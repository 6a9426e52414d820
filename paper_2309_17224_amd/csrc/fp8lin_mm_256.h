// The main loop of the 256-row matmul kernels (described in fp8lin_gemm.hip):
// one 256 x TN tile of A [M, K] . B [N, K]^T, K a multiple of 128, into the
// accumulators of a workgroup of 8 waves.  Internal, not part of the ABI.
#pragma once

#include "fp8lin_mm.h"

namespace fp8lin {
namespace {

constexpr int kBM = 256, kBN = 256, kBK = 128;
constexpr int kMainThreads = 512;      // 8 waves: two groups of four
constexpr int kTileBytes = kBM * kBK;  // one operand tile, 32 KiB
// LDS of the main loop: two A stages and three B stages (B tiles are copied two
// steps ahead).
constexpr int kSmemBytes = 2 * kTileBytes + 3 * kBN * kBK;

// Tile rows m0 .. m0 + 255 of A, n0 .. n0 + TN - 1 of B (TN = 64..256); wave w
// (group g = w / 4, quadrant sq = w % 4) gets rows (sq / 2) 128 + g 64 .. + 63
// and columns (sq % 2) TN/2 .. + TN/2 - 1: acc[i][j] is the 16 x 16 block (i, j)
// of those, lane l holding row l % 16, columns 4 (l / 16) .. + 3 of it.
// PAIR: B is two matrices of N rows each, one after the other, and a tile takes
// blocks of 16 rows from them in turn (pair_row), from row n0 / 2 on of each: a
// lane then holds the same four columns of both products in acc[i][2 j] and
// acc[i][2 j + 1].
// Rows past a matrix's edge are copies of its last one.
template <int FA, int FB, int TN, bool PAIR>
__device__ __forceinline__ void mm256_loop(uint8_t* __restrict__ smem, const uint8_t* __restrict__ A,
                                           const uint8_t* __restrict__ B, int M, int N, int K, int m0, int n0,
                                           v4f (&acc)[4][TN / 32]) {
    constexpr int kNbw = TN / 32;      // 16-column blocks per wave, B copies per loader wave
    constexpr int kBStage = TN * kBK;  // one B tile in LDS
    constexpr int kNf = 4 + kNbw;      // fragment pieces a wave reads per step
    constexpr int kNc = 8 + kNbw;      // copies a loader wave issues per stage
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    // group (0: waves 0-3, 1: waves 4-7) and quadrant; wave-uniform
    const int g = __builtin_amdgcn_readfirstlane(w >> 2), sq = __builtin_amdgcn_readfirstlane(w & 3);

    // Loaders: wave sq of group 0 fills rows [64 sq, 64 sq + 64) of the A tile, of
    // group 1 rows [TN/4 sq, TN/4 (sq + 1)) of the B tile, 8 rows per copy (voff[i] is
    // that of the group's own operand); lane -> row r = (first row) + 8 i + lane / 8
    // and physical chunk lane % 8, which holds logical chunk (lane % 8) ^
    // chunk_swz(r).  Rows past the matrix edge re-read the last row (their
    // outputs are not stored).  Offsets are relative to the tile's first row,
    // so they fit 32 bits for K < 2^22.
    const int lrow = lane >> 3;
    uint32_t voff[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = (g == 0 ? sq * 64 : sq * (TN / 4)) + i * 8 + lrow;
        const int src = g == 0 ? min(m0 + r, M - 1) - m0
                        : PAIR ? min(n0 / 2 + pair_row(r), N - 1) - n0 / 2
                               : min(n0 + r, N - 1) - n0;
        voff[i] = (uint32_t)(src * K + ((lane & 7) ^ chunk_swz(r)) * 16);
    }
    const uint8_t* baseA = A + (int64_t)m0 * K;
    const uint8_t* baseB = B + (int64_t)(PAIR ? n0 / 2 : n0) * K;
    const int64_t second = PAIR ? (int64_t)N * K : 0;  // from a row of the first matrix to the second's
    // LDS addresses of this wave's first loader rows (wave-uniform); copy d
    // < 8 fills A row group d, copy d >= 8 B row group d - 8.
    // LDS: A stages 0 and 1 at s * kTileBytes, B stages 0, 1 and 2 after them.
    const uint32_t lds_a = __builtin_amdgcn_readfirstlane(lds_addr(smem) + sq * 64 * kBK);
    const uint32_t lds_b = __builtin_amdgcn_readfirstlane(lds_addr(smem) + 2 * kTileBytes + sq * (TN / 4) * kBK);
    auto dma = [&](int d, int stage, int k0) {  // stage: of A for d < 8, of B for d >= 8
        // a copy's eight rows lie in one block of 16: which of the pair is wave-uniform
        const bool up = PAIR && d >= 8 && ((sq * (TN / 64) + ((d - 8) >> 1)) & 1);
        lds_dma16_s((d >= 8 ? baseB : baseA) + k0 + (up ? second : 0), voff[d & 7],
                    d >= 8 ? lds_b + (d - 8) * 8 * kBK + stage * kBStage : lds_a + d * 8 * kBK + stage * kTileBytes);
    };

    const int wr0 = (sq >> 1) * 128 + g * 64, wc0 = (sq & 1) * (TN / 2);
    const int frow = lane & 15, fg = lane >> 4;
    // byte offsets (within a 16-row block) of this lane's two fragment pieces
    const int fo0 = frow * kBK + (((2 * fg) ^ chunk_swz(frow)) << 4);
    const int fo1 = frow * kBK + (((2 * fg + 1) ^ chunk_swz(frow)) << 4);

#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kNbw; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    // Ping-pong pipeline.  Phases are separated by workgroup barriers; in
    // every phase one group issues MFMAs and the other loads:
    //   phase 1:        group 0 loads fragments of step 0
    //   phase 2k + 2:   group 0 MFMAs of step k,   group 1 loads step k
    //   phase 2k + 3:   group 0 loads step k + 1,  group 1 MFMAs of step k
    // A load phase reads all kNf fragment pieces of the wave's next step and
    // waits for them before the barrier.  A tile k sits in A stage k % 2, B
    // tile k in B stage k % 3.  Group 0 copies A tile k + 1 in its load phase
    // of step k (after both groups have read A tile k - 1 from that stage) and
    // waits for the copies at the end of its next MFMA phase.  Group 1 copies
    // B tile k + 2 in its load phase of step k (B tile k - 1 has been read by
    // then) and, before that phase's barrier, waits for B tile k + 1 — issued
    // one load phase earlier — but not for the copies it has just issued.
    // Steps 0 and 1 are copied before phase 1.  Every wave passes 2 nk + 1
    // barriers (group 1 passes one before its first load phase and none after
    // its last MFMA phase), so the groups stay in step.
    const int nk = K / kBK;
    if (nk > 0) {
        if (g == 0) {
#pragma unroll
            for (int d = 0; d < 8; ++d) dma(d, 0, 0);
            if (nk > 1) {
#pragma unroll
                for (int d = 0; d < 8; ++d) dma(d, 1, kBK);
                wait_vmcnt<8>();
            } else {
                wait_vmcnt<0>();
            }
        } else {
#pragma unroll
            for (int d = 8; d < kNc; ++d) dma(d, 0, 0);
            if (nk > 1) {
#pragma unroll
                for (int d = 8; d < kNc; ++d) dma(d, 1, kBK);
                wait_vmcnt<kNbw>();
            } else {
                wait_vmcnt<0>();
            }
        }
        ws_barrier();
        if (g == 1) ws_barrier();
    }
    v8i af[4], bf[kNbw];
    int bs = 0;  // k % 3: the B stage of step k
    for (int kt = 0; kt < nk; ++kt) {
        const uint8_t* sa = smem + (kt & 1) * kTileBytes + wr0 * kBK;
        const uint8_t* sb = smem + 2 * kTileBytes + bs * kBStage + wc0 * kBK;
        if (g == 0 && kt >= 1 && kt + 1 < nk) {
            // A tile of step kt + 1, the copies spread over the fragment reads
            const int st = (kt + 1) & 1, k1 = (kt + 1) * kBK;
#pragma unroll
            for (int q = 0; q < kNf; ++q) {
                if (q < 4) af[q] = ld_frag(sa + q * 16 * kBK, fo0, fo1);
                else bf[q - 4] = ld_frag(sb + (q - 4) * 16 * kBK, fo0, fo1);
                if (q < 8) dma(q, st, k1);
            }
#pragma unroll
            for (int d = kNf; d < 8; ++d) dma(d, st, k1);
        } else if (g == 1 && kt + 2 < nk) {
            // B tile of step kt + 2 into the stage B tile kt - 1 used
            const int st = bs == 0 ? 2 : bs - 1, k2 = (kt + 2) * kBK;
#pragma unroll
            for (int q = 0; q < kNf; ++q) {
                if (q < 4) af[q] = ld_frag(sa + q * 16 * kBK, fo0, fo1);
                else bf[q - 4] = ld_frag(sb + (q - 4) * 16 * kBK, fo0, fo1);
                if (q < kNbw) dma(8 + q, st, k2);
            }
        } else {
#pragma unroll
            for (int q = 0; q < kNf; ++q) {
                if (q < 4) af[q] = ld_frag(sa + q * 16 * kBK, fo0, fo1);
                else bf[q - 4] = ld_frag(sb + (q - 4) * 16 * kBK, fo0, fo1);
            }
        }
        if (g == 1) {  // B tile kt + 1 has landed (the copies just issued need not have)
            if (kt + 2 < nk) wait_vmcnt<kNbw>();
            else wait_vmcnt<0>();
        }
        bs = bs == 2 ? 0 : bs + 1;
        wait_lgkmcnt0();
        ws_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kNbw; ++j) {
                acc[i][j] = mfma16<FB, FA>(bf[j], af[i], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        if (g == 0) {
            wait_vmcnt<0>();
            ws_barrier();
        } else if (kt + 1 < nk) {
            ws_barrier();
        }
    }
}

}  // namespace
}  // namespace fp8lin
