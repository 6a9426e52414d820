// The feed-forward matmuls (fp8lin_ffn.hip) for outputs too small to fill the
// chip with 256 x 256 tiles, single tokens among them, for gfx950: the small
// tiles of fp8lin_gemm_stream.hip.  The partial sums of the waves are added
// through LDS in a fixed order as there; each wave then takes whole blocks of 16
// x 16 outputs (with kEpiGlu the two blocks of a pair), a lane four columns of a
// row.  The weight's stream bounds it where there are few rows (16 x 28672 x 8192 gated:
// 70 us, 6.7 TB/s; 1 x 4096 x 11008 with bias and residual: 12 us, 3.7 TB/s, since a 16 x 16
// tile has two stages of 16 KB on the way, half of each copies of the one row of
// activations: 4 MB of weights at a time over the chip), launches and latency where both sides
// are small (509 x 2048 x 768 backward with codes and bias gradient: 10 us, with the launch
// that finishes both 13).
#include "fp8lin_epilogue.h"
#include "fp8lin_mm_stream.h"

namespace fp8lin {
namespace {

template <int MODE>
struct Finish {
    using Args = Epi;
    static constexpr bool kPlain = false, kPair = MODE == kEpiGlu;

    template <int MB, int NB, int SLOTS>
    static __device__ __forceinline__ void finish(const Epi& e, const v4f* red, uint32_t* wmx, int m0, int n0) {
        constexpr int kFmt = epi_fwd(MODE) ? FP8_E4M3 : FP8_E5M2;
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, frow = lane & 15, fg = lane >> 4;
        const int sh = -(*e.ba + *e.bb);
        auto total = [&](int b, float (&y)[4]) {
            v4f sum = red[b * 64 + lane];
#pragma unroll
            for (int s = 1; s < SLOTS; ++s) sum += red[(s * MB * NB + b) * 64 + lane];
#pragma unroll
            for (int v = 0; v < 4; ++v) y[v] = ldexpf(sum[v], sh);
        };
        // Four codes of row m from column n on; transposed they are single bytes, of
        // sixteen rows side by side over the lanes.
        const int bq = e.q ? clamp_bias(*e.pred) : 0;
        uint32_t mag = 0;
        auto codes = [&](const float (&y)[4], int64_t m, int64_t n, int nv) {
            const uint32_t lo = pack_bf16x2(nv > 0 ? y[0] : 0.0f, nv > 1 ? y[1] : 0.0f);
            const uint32_t hi = pack_bf16x2(nv > 2 ? y[2] : 0.0f, nv > 3 ? y[3] : 0.0f);
            uint32_t c = cast4_bf16<kFmt>(lo, hi, bq);
            if (__builtin_expect(any_nan_bf16(lo, hi), 0)) {
                const uint32_t h[4] = {lo & 0xFFFFu, lo >> 16, hi & 0xFFFFu, hi >> 16};
                c = nan_patch<kFmt>(c, h);
            }
            mag = max(mag, max(max(lo & 0x7FFFu, (lo >> 16) & 0x7FFFu), max(hi & 0x7FFFu, (hi >> 16) & 0x7FFFu)));
            uint8_t* p = e.q + m * e.ldq + n;
            if (nv >= 4) *(u32_any*)p = c;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (v < nv) {
                    if (nv < 4) p[v] = (uint8_t)(c >> (8 * v));
                    if (e.qT) e.qT[(n + v) * e.ldqT + m] = (uint8_t)(c >> (8 * v));
                }
        };
        constexpr int kStep = kPair ? 2 : 1, kPerRow = NB / kStep;
        for (int b = w; b < MB * kPerRow; b += stream_threads(MB) / 64) {
            const int mb = b / kPerRow, nb = b % kPerRow;
            const int64_t m = m0 + mb * 16 + frow, n = n0 / kStep + nb * 16 + fg * 4;
            const int nv = (int)min((int64_t)4, e.N - n);
            float t[4], u[4], sa[4] = {}, sb[4] = {};
            total(mb * NB + nb * kStep, t);
            if (kPair) total(mb * NB + nb * kStep + 1, u);
            if (nv > 0 && m < e.M) {
                float y[4], x[4];
                epi_row<MODE, 4>(e, m, n, nv, t, u, sa, sb, y, x);
                if (e.q) {
                    codes(y, m, n, nv);
                    if (MODE == kEpiGluBwd) codes(x, m, e.N + n, nv);
                }
            }
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
        if (e.q) {  // the workgroup's largest output, for the exact bias
            const uint32_t wv = wave_max_u32(mag);
            if (lane == 0) wmx[w] = wv;
            __syncthreads();
            if (threadIdx.x == 0) {
                uint32_t b = 0;
#pragma unroll
                for (int v = 0; v < stream_threads(MB) / 64; ++v) b = max(b, wmx[v]);
                e.parts[blockIdx.x] = b;
                if (blockIdx.x == 0) *e.used = bq;
            }
        }
    }
};

template <int MODE, int MB, int NB>
void launch_one(const Epi& e, hipStream_t s) {
    const int64_t cols = MODE == kEpiGlu ? 2 * ((e.N + 15) / 16 * 16) : e.N;
    const int tm = (int)((e.M + 16 * MB - 1) / (16 * MB)), tn = (int)((cols + 16 * NB - 1) / (16 * NB));
    hipLaunchKernelGGL((gemm_nt_stream<epi_fa(MODE), FP8_E4M3, MB, NB, Finish<MODE>>), dim3((unsigned)(tm * tn)),
                       dim3(stream_threads(MB)), 0, s, e, tm, tn, tm == 1);
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
