// The main loop of the matmul kernels for any contraction length (described in
// fp8lin_gemm_ragged.hip): one BM x BN tile of A [M, K] . B [N, K]^T into the
// accumulators.  Internal, not part of the ABI.
#pragma once

#include "fp8lin_mm.h"

namespace fp8lin {
namespace {

constexpr int kRk = 128;  // bytes of k per step

// Bytes [k, k + 16) of a row of K bytes, zero from K on; reads only bytes of
// the row.  With K >= 16 one load ending at the row's end, moved down.
__device__ __forceinline__ uint4 ld16_tail(const uint8_t* row, int64_t k, int64_t K) {
    if (K < 16) {  // one or two loads that overlap: sixteen guarded bytes took 1.7 us
        if (k > 0) return make_uint4(0u, 0u, 0u, 0u);
        if (K >= 8) {
            const u32x2_any lo = *(const u32x2_any*)row, hi = *(const u32x2_any*)(row + K - 8);
            const uint64_t h = (hi.x | ((uint64_t)hi.y << 32)) >> 8 >> (8 * (15 - K));
            return make_uint4(lo.x, lo.y, (uint32_t)h, (uint32_t)(h >> 32));
        }
        if (K >= 4) {
            const uint32_t lo = *(const u32_any*)row, hi = *(const u32_any*)(row + K - 4);
            return make_uint4(lo, hi >> 8 >> (8 * (7 - K)), 0u, 0u);
        }
        const uint32_t b0 = row[0], b1 = row[min((int64_t)1, K - 1)], b2 = row[K - 1];
        return make_uint4(b0 | (K > 1 ? b1 << 8 : 0u) | (K > 2 ? b2 << 16 : 0u), 0u, 0u, 0u);
    }
    const int64_t at = min(k, K - 16);
    const int sh = (int)min(k - at, (int64_t)16) * 8;  // bits to drop
    return shr128(ld16_any(row + at), sh);
}

// Tile rows m0 .. of A and n0 .. of B; a workgroup of (BM / WT) (BN / WT) waves,
// wave w with the WT x WT outputs at row w / (BN / WT) WT, column w % (BN / WT)
// WT, laid out as in mm256_loop.  smem: 2 (BM + BN) kRk bytes of LDS, which every
// wave has finished reading on return.  PAIR: as in mm256_loop.
template <int FA, int FB, int BM, int BN, int WT, bool PAIR>
__device__ __forceinline__ void ragged_loop(uint8_t* smem, const uint8_t* A,
                                            const uint8_t* B, int64_t M, int64_t N, int64_t K, int64_t m0,
                                            int64_t n0, v4f (&acc)[WT / 16][WT / 16]) {
    constexpr int kNt = (BM / WT) * (BN / WT) * 64;
    constexpr int kRows = BM + BN, kStage = kRows * kRk;
    constexpr int kRpi = kNt / 8;      // rows per load of the workgroup (8 lanes a row)
    constexpr int kNc = kRows / kRpi;  // loads per thread and step
    constexpr int kB = WT / 16;        // 16-row blocks of a wave's sub-tile
    static_assert(kRows % kRpi == 0 && BM % kRpi == 0, "loader rows");
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;

    // loader: chunk tid % 8 of rows tid / 8 + i kRpi of the tile (A rows, then
    // B rows); rows past the matrix edge read the last row (not stored)
    const int lc = tid & 7, lr = tid >> 3;
    const uint8_t* row[kNc];
    uint32_t dst[kNc];
#pragma unroll
    for (int i = 0; i < kNc; ++i) {
        const int r = lr + i * kRpi;
        const int rb = r - BM;
        const int64_t nb = PAIR ? min(n0 / 2 + pair_row(rb), N - 1) + ((rb >> 4) & 1) * N : min(n0 + rb, N - 1);
        row[i] = i * kRpi < BM ? A + min(m0 + r, M - 1) * K : B + nb * K;
        dst[i] = r * kRk + ((lc ^ chunk_swz(r)) << 4);
    }
    const int nk = (int)((K + kRk - 1) / kRk);
    uint4 rg[kNc];
    auto load = [&](int kt) {
        const int64_t k = (int64_t)kt * kRk + lc * 16;
        if ((int64_t)(kt + 1) * kRk <= K) {
#pragma unroll
            for (int i = 0; i < kNc; ++i) rg[i] = ld16_any(row[i] + k);
        } else if (K % 16 == 0) {  // whole chunks, nothing to shift (1024 x 8 x 64: 4.6 us with)
#pragma unroll
            for (int i = 0; i < kNc; ++i) {
                const uint4 v = ld16_any(row[i] + min(k, K - 16));
                rg[i] = k < K ? v : make_uint4(0u, 0u, 0u, 0u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kNc; ++i) rg[i] = ld16_tail(row[i], k, K);
        }
    };
    auto store = [&](int kt) {
        uint8_t* d = smem + (kt & 1) * kStage;
#pragma unroll
        for (int i = 0; i < kNc; ++i) *(uint4*)(d + dst[i]) = rg[i];
    };

    const int wr0 = (w / (BN / WT)) * WT, wc0 = (w % (BN / WT)) * WT;
    const int frow = lane & 15, fg = lane >> 4;
    const int fo0 = frow * kRk + (((2 * fg) ^ chunk_swz(frow)) << 4);
    const int fo1 = frow * kRk + (((2 * fg + 1) ^ chunk_swz(frow)) << 4);
#pragma unroll
    for (int i = 0; i < kB; ++i)
#pragma unroll
        for (int j = 0; j < kB; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    if (nk > 0) {
        load(0);
        store(0);
        if (nk > 1) load(1);
    }
    wait_lgkmcnt0();
    ws_barrier();
    // step kt: write step kt + 1 (loaded during step kt - 1) into the other
    // stage, which every wave finished reading before the last barrier, issue
    // the loads of step kt + 2, multiply step kt
    for (int kt = 0; kt < nk; ++kt) {
        if (kt + 1 < nk) {
            store(kt + 1);
            if (kt + 2 < nk) load(kt + 2);
        }
        __builtin_amdgcn_sched_barrier(0);
        const uint8_t* sa = smem + (kt & 1) * kStage + wr0 * kRk;
        const uint8_t* sb = smem + (kt & 1) * kStage + (BM + wc0) * kRk;
        v8i af[kB], bf[kB];
#pragma unroll
        for (int i = 0; i < kB; ++i) af[i] = ld_frag(sa + i * 16 * kRk, fo0, fo1);
#pragma unroll
        for (int j = 0; j < kB; ++j) bf[j] = ld_frag(sb + j * 16 * kRk, fo0, fo1);
#pragma unroll
        for (int i = 0; i < kB; ++i)
#pragma unroll
            for (int j = 0; j < kB; ++j) acc[i][j] = mfma16<FB, FA>(bf[j], af[i], acc[i][j]);
        wait_lgkmcnt0();
        ws_barrier();
    }
}

}  // namespace
}  // namespace fp8lin
