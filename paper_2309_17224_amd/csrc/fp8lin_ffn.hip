// The choice of kernel for the feed-forward matmuls (fp8lin_ffn.h), the column sums
// that their backward epilogues leave in parts, and the quantise of their output.
#include "fp8lin_mm.h"
#include "fp8lin_sums.h"
#include "fp8lin_vals.h"

namespace fp8lin {
namespace {

// ------------------------------------------------------------ column sums
__global__ __launch_bounds__(1024) void sums_finish_kernel(const float* __restrict__ part, int rows, int64_t cols,
                                                           void* out0, int64_t n0, void* out1, int dt) {
    __shared__ float red[16][64];
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < cols; c0 += (int64_t)gridDim.x * 64)
        sum_rows64<16>(red, part, rows, cols, c0, out0, n0, out1, dt);
}

// The same where there are many rows of few columns: 32 columns a workgroup, 32 sums of
// every 32nd row each.  512 rows of 1536 sums (layer norm of 4096 x 768, its two launches)
// 13.4 -> 12.0 us, of 4096 sums (4096 x 2048) 19.8 -> 18.3; 16 columns are slower, 64-byte
// runs being half a line.
constexpr int kFineRows = 256, kFineCols = 8192;
__global__ __launch_bounds__(1024) void sums_finish_fine_kernel(const float* __restrict__ part, int rows, int64_t cols,
                                                                void* out0, int64_t n0, void* out1, int dt) {
    constexpr int C = 32, kS = 1024 / C;
    __shared__ float red[16][C];
    const int c = threadIdx.x % C, s = threadIdx.x / C;
    const int64_t col = (int64_t)blockIdx.x * C + c;
    const float* p = part + min(col, cols - 1);
    float v = 0.0f;
    for (int r0 = s; r0 < rows; r0 += 8 * kS) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = p[(int64_t)min(r0 + kS * k, rows - 1) * cols];
#pragma unroll
        for (int k = 0; k < 8; ++k) v += r0 + kS * k < rows ? x[k] : 0.0f;
    }
#pragma unroll
    for (int off = C; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) < C) red[threadIdx.x >> 6][c] = v;
    __syncthreads();
    void* out = col < n0 ? out0 : out1;
    if (s == 0 && col < cols && out) {
        v = red[0][c];
#pragma unroll
        for (int k = 1; k < 16; ++k) v += red[k][c];
        const int64_t at = col < n0 ? col : col - n0;
        if (dt == FP8_DT_BF16) ((uint16_t*)out)[at] = (uint16_t)(pack_bf16x2(v, 0.0f) & 0xFFFFu);
        else ((float*)out)[at] = v;
    }
}

// ------------------------------------------------------------ transposed codes
// qT [cols, rows] = q [rows, cols]^T, bytes: a workgroup's 256 rows x 128 columns
// through LDS, so that both sides move 16-byte pieces of whole runs: memory bounds it
// (4096 x 22016: 31 us, 5.8 TB/s; the whole quantise after the matmul instead of the
// codes in its epilogue and this: 286 instead of 263 us).  A column is 256
// bytes of LDS, its 16-byte chunk c at chunk c ^ swz(column).
constexpr int kTr = 256, kTc = 128;

__global__ __launch_bounds__(256) void transpose_codes_kernel(const uint8_t* __restrict__ q, int64_t ldq,
                                                              uint8_t* __restrict__ qT, int64_t ldqT, int64_t rows,
                                                              int64_t cols) {
    __shared__ __attribute__((aligned(16))) uint8_t cs[kTc * kTr];
    auto swz = [](int col) { return (col ^ (col >> 4)) & 15; };
    const int64_t tiles_m = (rows + kTr - 1) / kTr;
    const int64_t m0 = blockIdx.x % tiles_m * kTr, n0 = blockIdx.x / tiles_m * kTc;
    const int mr = (int)min((int64_t)kTr, rows - m0), nc = (int)min((int64_t)kTc, cols - n0);
    uint4 v[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // four rows, sixteen columns a turn
        const int i = threadIdx.x + 256 * h, r = (i >> 3) * 4, c = (i & 7) * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[h][k] = make_uint4(0u, 0u, 0u, 0u);
            const uint8_t* p = q + (m0 + r + k) * ldq + n0 + c;
            if (r + k < mr && c + 16 <= nc) {
                v[h][k] = ld_stream(p);
            } else if (r + k < mr && c < nc) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int b = 0; b < 16; ++b) w[b >> 2] |= c + b < nc ? (uint32_t)p[b] << (8 * (b & 3)) : 0u;
                v[h][k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = threadIdx.x + 256 * h, r = (i >> 3) * 4, c = (i & 7) * 16;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint32_t t[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = g == 0 ? v[h][k].x : g == 1 ? v[h][k].y : g == 2 ? v[h][k].z : v[h][k].w;
            transpose4(t);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int n = c + 4 * g + k;
                *(uint32_t*)(cs + n * kTr + (((r >> 4) ^ swz(n)) << 4) + (r & 15)) = t[k];
            }
        }
    }
    __syncthreads();
    const int c16 = threadIdx.x & 15, left = mr - c16 * 16;
    for (int n = threadIdx.x >> 4; n < nc; n += 16) {
        const uint4 x = *(const uint4*)(cs + n * kTr + ((c16 ^ swz(n)) << 4));
        uint8_t* p = qT + (n0 + n) * ldqT + m0 + c16 * 16;
        if (left >= 16) {
            st16_any(p, x);
        } else {
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int b = 0; b < 16; ++b)
                if (b < left) p[b] = (uint8_t)(w[b >> 2] >> (8 * (b & 3)));
        }
    }
}

}  // namespace

// Rows of partial sums up to which the launch that checks the codes' bias adds them up too
// (it costs a launch less and has fewer waves: 32 rows of a 509 x 2048 output 14.1 -> 13.1 us
// the whole call, 256 rows of 16384 x 4096 154.9 -> 154.4; 512 rows 156.0 -> 159.4).
constexpr int kJoinRows = 256;

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
    if (rows > kFineRows && cols <= kFineCols) {
        hipLaunchKernelGGL(sums_finish_fine_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(1024), 0, s, part, (int)rows,
                           cols, out0, n0, out1, dt);
        return hip_status();
    }
    hipLaunchKernelGGL(sums_finish_kernel, dim3((unsigned)sum_blocks(cols)), dim3(1024), 0, s, part, (int)rows, cols,
                       out0, n0, out1, dt);
    return hip_status();
}

int32_t launch_epilogue_mm(int mode, Epi& e, const FusedQuant* fq, int64_t ws_words, uint8_t* qT, int64_t ldqT,
                           hipStream_t s) {
    const MmRoute r = epi_route(mode, e.M, e.N, e.K);
    const int64_t cols = mode == kEpiGluBwd ? 2 * e.N : e.N;
    // 32-bit offsets within a wave's rows (64) and, for transposed codes, columns (128)
    constexpr int64_t kFar = 1 << 22;
    e.fast = e.out_dt == FP8_DT_BF16 && e.ldo <= kFar && e.ldres <= kFar && e.ldkeep <= kFar && e.ldz <= kFar;
    e.q = nullptr;
    const int64_t bc = epi_b_cols(mode, e.N);
    int64_t blocks;
    if (r.kernel == kMmStream) {
        blocks = stream_workgroups(e.M, bc, r.mb, r.nb);
    } else if (r.kernel == kMm256) {
        const int tm = (int)((e.M + 255) / 256), tn = (int)((bc + 255) / 256);
        int ndp, tw, tn2;
        mm256_split(tm, tn, bc, ndp, tw, tn2);
        blocks = (int64_t)tm * (ndp + tn2);
    } else {
        blocks = ((e.M + 255) / 256) * ((bc + 127) / 128);  // at most 128 of the smaller tiles are four times as many
    }
    if (blocks > UINT32_MAX / 512) return FP8_ENOTSUP;  // workgroups of up to 512 threads; a launch has fewer than 2^32
    // Codes from the epilogue, with the predicted bias: where each workgroup finds a word
    // for its largest output, in the format of the matmul that reads them.
    const bool casts = r.kernel == kMmStream ||
                       (r.kernel == kMm256 && e.fast && e.N % 8 == 0 && fq && fq->ldq <= kFar && ldqT <= kFar);
    if (fq && fq->pred && e.out_dt == FP8_DT_BF16 && casts && 1 + blocks <= ws_words &&
        fq->fmt == (mode == kEpiAct || mode == kEpiGlu ? FP8_E4M3 : FP8_E5M2)) {
        e.pred = fq->pred, e.used = (int32_t*)fq->ws, e.parts = fq->ws + 1;
        e.q = fq->q, e.ldq = fq->ldq, e.qT = qT, e.ldqT = ldqT;
    }
    if (r.kernel == kMmStream) launch_ffn_small(mode, r.mb, r.nb, e, s);
    else if (mode == kEpiAct) launch_ffn_act(r.kernel == kMmRagged, e, s);
    else if (mode == kEpiGlu) launch_ffn_glu(r.kernel == kMmRagged, e, s);
    else if (mode == kEpiActBwd) launch_ffn_act_bwd(r.kernel == kMmRagged, e, s);
    else launch_ffn_glu_bwd(r.kernel == kMmRagged, e, s);
    int32_t st = hip_status();
    // The column sums, with the check of the codes' bias in one launch where both are due.
    ColumnSums sums{e.sums, e.sums ? (int)epi_sum_rows(mode, e.M, e.N, e.K) : 0, e.db_dt, cols, e.db};
    const bool join = e.q && e.sums && sums.rows <= kJoinRows;
    if (st == FP8_OK && e.sums && !join)
        st = launch_sums_finish(e.sums, sums.rows, cols, e.db, cols, nullptr, e.db_dt, s);
    if (st != FP8_OK || !fq) return st;
    if (e.q) {
        // The codes of both gradients of a gated block's tile, transposed, are 128 KB, and
        // whole rows of eight waves staged another 64 (half rows would leave room): from the
        // codes, once they are final.
        const bool apart = qT && mode == kEpiGluBwd && r.kernel == kMm256;
        st = launch_quant_check(e.out, FP8_DT_BF16, e.M, cols, e.ldo, fq->fmt, fq->margin, fq->ws + 1, (int)blocks,
                                (const int32_t*)fq->ws, fq->bias, fq->amax_bits, fq->flags, fq->q, fq->ldq,
                                apart ? nullptr : qT, apart ? 0 : ldqT, s, join ? &sums : nullptr);
        if (st != FP8_OK || !apart) return st;
        hipLaunchKernelGGL(transpose_codes_kernel, dim3((unsigned)((e.M + kTr - 1) / kTr * ((cols + kTc - 1) / kTc))),
                           dim3(256), 0, s, fq->q, fq->ldq, qT, ldqT, e.M, cols);
        return hip_status();
    }
    return launch_quantise(e.out, e.out_dt, e.M, cols, e.ldo, fq->fmt, fq->margin, fq->pred, fq->bias, fq->amax_bits,
                           fq->flags, fq->q, fq->ldq, qT, ldqT, fq->ws, s);
}

}  // namespace fp8lin
