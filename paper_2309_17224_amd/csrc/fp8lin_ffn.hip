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
#include "fp8lin_epilogue.h"
#include "fp8lin_mm_256.h"
#include "fp8lin_mm_ragged.h"

namespace fp8lin {
namespace {

constexpr int pow2_up(int n) { return n <= 1 ? 1 : 2 * pow2_up((n + 1) / 2); }

// The epilogue of one wave: MBLK x NBLK blocks of 16 x 16 sums (laid out as in
// mm256_loop) of rows m0 .., columns n0 .. of the output (with kEpiGlu NBLK / 2
// blocks of columns of each projection); ep: 32 rows of LDS of its own; srow: its
// row of the column sums.
template <int MODE, int MBLK, int NBLK>
__device__ __forceinline__ void wave_epilogue(const Epi& e, uint8_t* ep, const v4f (&acc)[MBLK][NBLK], int64_t m0,
                                              int64_t n0, int64_t srow) {
    constexpr bool kPair = MODE == kEpiGlu, kBwd = !epi_fwd(MODE);
    constexpr int kRow = NBLK * 64 + 16;              // staging row, bytes
    constexpr int kOct = kPair ? NBLK : 2 * NBLK;     // eights of columns in a row
    constexpr int kLpr = pow2_up(kOct), kRpp = 64 / kLpr;  // lanes a row, rows a pass
    static_assert(MBLK % 2 == 0 && (!kPair || NBLK % 2 == 0) && kRpp <= 32, "blocks of a wave");
    const int lane = threadIdx.x & 63, frow = lane & 15, fg = lane >> 4;
    const int sh = -(*e.ba + *e.bb);
    const int oct = lane & (kLpr - 1), r0 = lane / kLpr;
    const int64_t n = n0 + 8 * oct;
    const int nv = oct < kOct ? (int)min((int64_t)8, e.N - n) : 0;
    const int at = kPair ? (oct >> 1) * 128 + (oct & 1) * 32 : oct * 32;
    float sa[8] = {}, sb[8] = {};
#pragma unroll
    for (int i2 = 0; i2 < MBLK / 2; ++i2) {
#pragma unroll
        for (int ii = 0; ii < 2; ++ii)
#pragma unroll
            for (int j = 0; j < NBLK; ++j) {
                const v4f a = acc[2 * i2 + ii][j];
                *(float4*)(ep + (ii * 16 + frow) * kRow + (j * 16 + 4 * fg) * 4) =
                    make_float4(ldexpf(a[0], sh), ldexpf(a[1], sh), ldexpf(a[2], sh), ldexpf(a[3], sh));
            }
#pragma unroll 1
        for (int p = 0; p < 32 / kRpp; ++p) {
            const int row = p * kRpp + r0;
            const int64_t m = m0 + i2 * 32 + row;
            if (nv <= 0 || m >= e.M) continue;
            const uint8_t* src = ep + row * kRow + at;
            const float4 t0 = *(const float4*)src, t1 = *(const float4*)(src + 16);
            float t[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w}, u[8];
            if (kPair) {
                const float4 u0 = *(const float4*)(src + 64), u1 = *(const float4*)(src + 80);
                const float v[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
#pragma unroll
                for (int k = 0; k < 8; ++k) u[k] = v[k];
            }
            epi_row<MODE, 8>(e, m, n, nv, t, u, sa, sb);
        }
    }
    if (kBwd && e.sums) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int off = kLpr; off < 64; off <<= 1) {
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
}

// ------------------------------------------------------------ 256-row tiles
// Grid, tiles and the narrower last round as gemm_nt_256, over the columns of B
// (kEpiGlu: of both matrices, in blocks of 16 in turn).
template <int MODE, int TN>
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
    static_assert(8 * 32 * (TN * 2 + 16) <= kSmemBytes, "LDS budget");
    wave_epilogue<MODE, 4, TN / 32>(e, smem + w * 32 * (TN * 2 + 16), acc, m0 + wr0, (n0 + wc0) / (kPair ? 2 : 1),
                                    4 * tm + wr0 / 64);
}

template <int MODE, int TN2>
__global__ __launch_bounds__(kMainThreads) void ffn_256(Epi e, int tiles_m, int tiles_n, int g1, int tiles_n2) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kSmemBytes];
    const int b = blockIdx.x;
    if (TN2 == 0 || b < g1) ffn_tile<MODE, 256>(smem, b, TN2 == 0 ? (int)gridDim.x : g1, e, tiles_m, tiles_n, 0);
    else ffn_tile<MODE, (TN2 > 0 ? TN2 : 256)>(smem, b - g1, (int)gridDim.x - g1, e, tiles_m, tiles_n2, tiles_n * kBN);
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
    wave_epilogue<MODE, WT / 16, WT / 16>(e, smem + w * kEpWave, acc, m0 + wr0, (n0 + wc0) / (kPair ? 2 : 1),
                                          (m0 + wr0) / WT);
}

// ------------------------------------------------------------ column sums
// out[c] = sum of the rows of part [rows, cols], in order within each of 16
// slices of them, then over the slices: 16 columns a workgroup.  Columns from n0
// on go to out1.
__global__ __launch_bounds__(256) void sums_finish_kernel(const float* __restrict__ part, int rows, int64_t cols,
                                                          void* out0, int64_t n0, void* out1, int dt) {
    __shared__ float red[16][17];
    const int c = threadIdx.x & 15, s = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + c;
    float v = 0.0f;
    if (col < cols)
        for (int r = s; r < rows; r += 16) v += part[(int64_t)r * cols + col];
    red[s][c] = v;
    __syncthreads();
    if (s == 0 && col < cols) {
        v = red[0][c];
#pragma unroll
        for (int k = 1; k < 16; ++k) v += red[k][c];
        void* out = col < n0 ? out0 : out1;
        const int64_t at = col < n0 ? col : col - n0;
        if (!out) return;
        if (dt == FP8_DT_BF16) ((uint16_t*)out)[at] = (uint16_t)f32_to_bf16_rne(v);
        else ((float*)out)[at] = v;
    }
}

// Columns of the matmul's B over all tiles: with kEpiGlu the blocks of 16 of both
// matrices, the last one filled up.
int64_t b_cols(int mode, int64_t N) { return mode == kEpiGlu ? 2 * ((N + 15) / 16 * 16) : N; }

bool big_tiles(int64_t M, int64_t N) { return ((M + 255) / 256) * ((N + 127) / 128) >= 128; }

template <int MODE>
void launch_mode(const Epi& e, const MmRoute& r, hipStream_t s) {
    const int64_t cols = b_cols(MODE, e.N);
    if (r.kernel == kMmRagged) {
        if (big_tiles(e.M, cols)) {
            const int tm = (int)((e.M + 255) / 256), tn = (int)((cols + 127) / 128);
            hipLaunchKernelGGL((ffn_ragged<MODE, 256, 128, 64>), dim3((unsigned)((int64_t)tm * tn)), dim3(512), 0, s, e, tm, tn);
        } else {
            const int tm = (int)((e.M + 63) / 64), tn = (int)((cols + 63) / 64);
            hipLaunchKernelGGL((ffn_ragged<MODE, 64, 64, 32>), dim3((unsigned)((int64_t)tm * tn)), dim3(256), 0, s, e, tm, tn);
        }
        return;
    }
    const int tiles_m = (int)((e.M + kBM - 1) / kBM), tiles_n = (int)((cols + kBN - 1) / kBN);
    int ndp, tw, tn2;
    mm256_split(tiles_m, tiles_n, cols, ndp, tw, tn2);
    const int g1 = tiles_m * ndp;
    const dim3 grid(g1 + tiles_m * tn2), block(kMainThreads);
    if (tw == 64) hipLaunchKernelGGL((ffn_256<MODE, 64>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);
    else if (tw == 128) hipLaunchKernelGGL((ffn_256<MODE, 128>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);
    else if (tw == 192) hipLaunchKernelGGL((ffn_256<MODE, 192>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);
    else hipLaunchKernelGGL((ffn_256<MODE, 0>), grid, block, 0, s, e, tiles_m, ndp, g1, tn2);
}

}  // namespace

MmRoute epi_route(int mode, int64_t M, int64_t N, int64_t K) {
    return mm_route(M, b_cols(mode, N), K, false, mode == kEpiGlu);
}

int64_t epi_sum_rows(int mode, int64_t M, int64_t N, int64_t K) {
    const MmRoute r = epi_route(mode, M, N, K);
    if (r.kernel == kMmStream) return (M + 15) / 16;
    if (r.kernel == kMm256 || big_tiles(M, b_cols(mode, N))) return 4 * ((M + 255) / 256);
    return 2 * ((M + 63) / 64);
}

int32_t launch_sums_finish(const float* part, int64_t rows, int64_t cols, void* out0, int64_t n0, void* out1, int dt,
                           hipStream_t s) {
    hipLaunchKernelGGL(sums_finish_kernel, dim3((unsigned)((cols + 15) / 16)), dim3(256), 0, s, part, (int)rows, cols,
                       out0, n0, out1, dt);
    return hip_status();
}

int32_t launch_epilogue_mm(int mode, const Epi& e, hipStream_t s) {
    const MmRoute r = epi_route(mode, e.M, e.N, e.K);
    if (r.kernel == kMmStream) launch_ffn_small(mode, r.mb, r.nb, e, s);
    else if (mode == kEpiAct) launch_mode<kEpiAct>(e, r, s);
    else if (mode == kEpiGlu) launch_mode<kEpiGlu>(e, r, s);
    else if (mode == kEpiActBwd) launch_mode<kEpiActBwd>(e, r, s);
    else launch_mode<kEpiGluBwd>(e, r, s);
    return hip_status();
}

}  // namespace fp8lin
