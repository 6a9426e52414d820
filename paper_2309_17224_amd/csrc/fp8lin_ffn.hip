// The choice of kernel for the feed-forward matmuls (fp8lin_ffn.h), the column sums
// that their backward epilogues leave in parts, and the quantise of their output.
#include "fp8lin_mm.h"

namespace fp8lin {
namespace {

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

}  // namespace

int64_t epi_b_cols(int mode, int64_t N) { return mode == kEpiGlu ? 2 * ((N + 15) / 16 * 16) : N; }

bool epi_big_tiles(int64_t M, int64_t cols) { return ((M + 255) / 256) * ((cols + 127) / 128) >= 128; }

MmRoute epi_route(int mode, int64_t M, int64_t N, int64_t K) {
    return mm_route(M, epi_b_cols(mode, N), K, false, mode == kEpiGlu);
}

int64_t epi_sum_rows(int mode, int64_t M, int64_t N, int64_t K) {
    const MmRoute r = epi_route(mode, M, N, K);
    if (r.kernel == kMmStream) return (M + 15) / 16;
    if (r.kernel == kMm256 || epi_big_tiles(M, epi_b_cols(mode, N))) return 4 * ((M + 255) / 256);
    return 2 * ((M + 63) / 64);
}

int32_t launch_sums_finish(const float* part, int64_t rows, int64_t cols, void* out0, int64_t n0, void* out1, int dt,
                           hipStream_t s) {
    hipLaunchKernelGGL(sums_finish_kernel, dim3((unsigned)((cols + 15) / 16)), dim3(256), 0, s, part, (int)rows, cols,
                       out0, n0, out1, dt);
    return hip_status();
}

int32_t launch_epilogue_mm(int mode, Epi& e, const FusedQuant* fq, uint8_t* qT, int64_t ldqT, hipStream_t s) {
    const MmRoute r = epi_route(mode, e.M, e.N, e.K);
    const int64_t cols = mode == kEpiGluBwd ? 2 * e.N : e.N;
    // 32-bit offsets within a wave's rows (64) and, for transposed codes, columns (128)
    constexpr int64_t kFar = 1 << 22;
    e.fast = e.out_dt == FP8_DT_BF16 && e.ldo <= kFar && e.ldres <= kFar && e.ldkeep <= kFar && e.ldz <= kFar;
    e.q = nullptr;
    int parts = 0;
    if (fq && fq->pred && r.kernel == kMm256 && e.fast && e.N % 8 == 0 && fq->ldq <= kFar && ldqT <= kFar &&
        fq->fmt == (mode == kEpiAct || mode == kEpiGlu ? FP8_E4M3 : FP8_E5M2)) {
        const int64_t bc = epi_b_cols(mode, e.N);
        const int tm = (int)((e.M + 255) / 256), tn = (int)((bc + 255) / 256);
        int ndp, tw, tn2;
        mm256_split(tm, tn, bc, ndp, tw, tn2);
        parts = tm * (ndp + tn2);
        if (1 + parts <= gemm_quantise_ws_words(e.M, cols)) {
            e.pred = fq->pred, e.used = (int32_t*)fq->ws, e.parts = fq->ws + 1;
            e.q = fq->q, e.ldq = fq->ldq, e.qT = qT, e.ldqT = ldqT;
        }
    }
    if (r.kernel == kMmStream) launch_ffn_small(mode, r.mb, r.nb, e, s);
    else if (mode == kEpiAct) launch_ffn_act(r.kernel == kMmRagged, e, s);
    else if (mode == kEpiGlu) launch_ffn_glu(r.kernel == kMmRagged, e, s);
    else if (mode == kEpiActBwd) launch_ffn_act_bwd(r.kernel == kMmRagged, e, s);
    else launch_ffn_glu_bwd(r.kernel == kMmRagged, e, s);
    int32_t st = hip_status();
    if (st == FP8_OK && e.sums)
        st = launch_sums_finish(e.sums, epi_sum_rows(mode, e.M, e.N, e.K), cols, e.db, cols, nullptr, e.db_dt, s);
    if (st != FP8_OK || !fq) return st;
    if (e.q)
        return launch_quant_check(e.out, FP8_DT_BF16, e.M, cols, e.ldo, fq->fmt, fq->margin, fq->ws + 1, parts,
                                  (const int32_t*)fq->ws, fq->bias, fq->amax_bits, fq->flags, fq->q, fq->ldq, qT, ldqT, s);
    return launch_quantise(e.out, e.out_dt, e.M, cols, e.ldo, fq->fmt, fq->margin, fq->pred, fq->bias, fq->amax_bits,
                           fq->flags, fq->q, fq->ldq, qT, ldqT, fq->ws, s);
}

}  // namespace fp8lin
