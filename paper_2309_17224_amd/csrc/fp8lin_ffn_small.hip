// The feed-forward matmuls (fp8lin_ffn.hip) for outputs too small to fill the
// chip with 256 x 256 tiles, single tokens among them, for gfx950: the small
// tiles of fp8lin_gemm_stream.hip.  The partial sums of the waves are added
// through LDS in a fixed order as there; each wave then takes whole blocks of 16
// x 16 outputs (with kEpiGlu the two blocks of a pair), a lane four columns of a
// row.
#include "fp8lin_epilogue.h"
#include "fp8lin_mm_stream.h"

namespace fp8lin {
namespace {

template <int MODE, int MB, int NB>
__global__ __launch_bounds__(stream_threads(MB)) void ffn_small(Epi e, int tiles_m, int tiles_n, int nt) {
    using T = StreamTile<MB, NB>;
    constexpr bool kPair = MODE == kEpiGlu;
    constexpr int kSlots = T::kSlots, kNbw = T::kNbw, kMbw = T::kMbw;
    static_assert(kSlots * MB * NB * 1024 <= kSlBuf * T::kStage && (!kPair || NB % 2 == 0), "LDS budget");
    __shared__ __attribute__((aligned(1024))) uint8_t sm[kSlBuf * T::kStage];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int x = blockIdx.x & 7, per = gridDim.x >> 3, rem = gridDim.x & 7;
    const int tile = x * per + min(x, rem) + (blockIdx.x >> 3);
    int tm = tile % tiles_m, tn = tile / tiles_m;
    if (kSlots == 1) tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * (16 * MB), n0 = tn * (16 * NB);
    const int frow = lane & 15, fg = lane >> 4;
    v4f acc[kMbw][kNbw];
    stream_loop<epi_fa(MODE), FP8_E4M3, MB, NB, kPair>(sm, e.A, e.B, (int)e.M, (int)e.N, (int)e.K, m0, n0, nt, acc);
    v4f* red = (v4f*)sm;  // [slot][16-row block][16-column block][lane]
    if (w < 4) {
        const int slot = w % kSlots, part = w / kSlots;
        const int nb0 = part % T::kWn * kNbw, mb0 = part / T::kWn * kMbw;  // this wave's blocks of the tile
#pragma unroll
        for (int i = 0; i < kMbw; ++i)
#pragma unroll
            for (int j = 0; j < kNbw; ++j) red[((slot * MB + mb0 + i) * NB + nb0 + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    const int sh = -(*e.ba + *e.bb);
    auto total = [&](int b, float (&y)[4]) {
        v4f sum = red[b * 64 + lane];
#pragma unroll
        for (int s = 1; s < kSlots; ++s) sum += red[(s * MB * NB + b) * 64 + lane];
#pragma unroll
        for (int v = 0; v < 4; ++v) y[v] = ldexpf(sum[v], sh);
    };
    constexpr int kStep = kPair ? 2 : 1, kPerRow = NB / kStep;
    for (int b = w; b < MB * kPerRow; b += stream_threads(MB) / 64) {
        const int mb = b / kPerRow, nb = b % kPerRow;
        const int64_t m = m0 + mb * 16 + frow, n = n0 / kStep + nb * 16 + fg * 4;
        const int nv = (int)min((int64_t)4, e.N - n);
        float t[4], u[4], sa[4] = {}, sb[4] = {};
        total(mb * NB + nb * kStep, t);
        if (kPair) total(mb * NB + nb * kStep + 1, u);
        if (nv > 0 && m < e.M) epi_row<MODE, 4>(e, m, n, nv, t, u, sa, sb);
        if (!epi_fwd(MODE) && e.sums) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) {
                    sa[v] += __shfl_xor(sa[v], off, 64);
                    if (MODE == kEpiGluBwd) sb[v] += __shfl_xor(sb[v], off, 64);
                }
            if (frow == 0 && m < e.M) {
                float* s = e.sums + (m >> 4) * e.sum_cols + n;
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (v < nv) {
                        s[v] = sa[v];
                        if (MODE == kEpiGluBwd) s[e.N + v] = sb[v];
                    }
            }
        }
    }
}

template <int MODE, int MB, int NB>
void launch_one(const Epi& e, hipStream_t s) {
    const int64_t cols = MODE == kEpiGlu ? 2 * ((e.N + 15) / 16 * 16) : e.N;
    const int tm = (int)((e.M + 16 * MB - 1) / (16 * MB)), tn = (int)((cols + 16 * NB - 1) / (16 * NB));
    hipLaunchKernelGGL((ffn_small<MODE, MB, NB>), dim3((unsigned)(tm * tn)), dim3(stream_threads(MB)), 0, s, e, tm, tn,
                       tm == 1);
}

template <int MODE>
void launch_t(int mb, int nb, const Epi& e, hipStream_t s) {
#define FP8LIN_FFN_CASE(MB, NB)                                  \
    if constexpr (MODE != kEpiGlu || NB % 2 == 0)                \
        if (mb == MB && nb == NB) return launch_one<MODE, MB, NB>(e, s);
    FP8LIN_STREAM_TILES(FP8LIN_FFN_CASE)
#undef FP8LIN_FFN_CASE
}

}  // namespace

void launch_ffn_small(int mode, int mb, int nb, const Epi& e, hipStream_t s) {
    if (mode == kEpiAct) launch_t<kEpiAct>(mb, nb, e, s);
    else if (mode == kEpiGlu) launch_t<kEpiGlu>(mb, nb, e, s);
    else if (mode == kEpiActBwd) launch_t<kEpiActBwd>(mb, nb, e, s);
    else launch_t<kEpiGluBwd>(mb, nb, e, s);
}

}  // namespace fp8lin
