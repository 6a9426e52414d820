// The main loop of the small-tile matmul kernels (described in
// fp8lin_gemm_stream.hip): one tile of 16 MB x 16 NB outputs of A [M, K] . B [N,
// K]^T, K a multiple of 128, into the accumulators of a workgroup's first four
// waves, which still hold partial sums over k.  Internal, not part of the ABI.
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

template <int MB, int NB>
struct StreamTile {
    static constexpr int kRowsB = 16 * NB, kRows = 16 * (MB + NB);
    static constexpr int kKC = stream_kc(MB, NB);
    static constexpr int kStage = kRows * kKC, kCpr = kKC / 16, kRpi = 64 / kCpr;  // chunks per row, rows per copy
    static constexpr int kNiw = kRows / kRpi / 4;                                  // copies per wave and stage
    static constexpr int kSlots = kKC / 128;                                       // slices of a stage's k
    static constexpr int kWn = kSlots == 4 ? 1 : 2, kWm = kSlots == 1 ? 2 : 1;     // waves over the tile's columns, rows
    static constexpr int kNbw = NB / kWn, kMbw = MB / kWm;
    static_assert(kRows % (4 * kRpi) == 0 && NB % kWn == 0 && MB % kWm == 0, "tile split");
    static_assert(kSlBuf * kStage <= 160 * 1024, "LDS budget");
};

// Tile rows m0 .. of A and n0 .. of B; wave w < 4 gets the k slice slot = w %
// kSlots of kMbw x kNbw blocks of 16 x 16: rows from block part / kWn * kMbw,
// columns from part % kWn * kNbw on (part = w / kSlots), laid out as in
// mm256_loop.  nt: B's rows are read by no other workgroup.  sm: kSlBuf * kStage
// bytes of LDS, which every wave has finished reading on return.
// PAIR: as in mm256_loop (NB even).
template <int FA, int FB, int MB, int NB, bool PAIR>
__device__ __forceinline__ void stream_loop(uint8_t* __restrict__ sm, const uint8_t* __restrict__ A,
                                            const uint8_t* __restrict__ B, int M, int N, int K, int m0, int n0, int nt,
                                            v4f (&acc)[StreamTile<MB, NB>::kMbw][StreamTile<MB, NB>::kNbw]) {
    using T = StreamTile<MB, NB>;
    constexpr int kRowsB = T::kRowsB, kKC = T::kKC, kStage = T::kStage, kCpr = T::kCpr, kRpi = T::kRpi, kNiw = T::kNiw;
    constexpr int kSlots = T::kSlots, kWn = T::kWn, kNbw = T::kNbw, kMbw = T::kMbw;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
                        : PAIR      ? min(n0 / 2 + pair_row(r), N - 1) - n0 / 2
                                    : min(n0 + r, N - 1) - n0;
        voff[t] = (uint32_t)(src * K + ((lchunk ^ swz(r)) << 4));
    }
    const uint8_t* baseA = A + (int64_t)m0 * K;
    const uint8_t* baseB = B + (int64_t)(PAIR ? n0 / 2 : n0) * K;
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
            const uint8_t* b = baseB + (PAIR && ((d * kRpi >> 4) & 1) ? (int64_t)N * K : 0);
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
}

}  // namespace
}  // namespace fp8lin
