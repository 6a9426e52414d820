// The paged key/value cache of the decoder layer for gfx950: the write of new
// tokens (rotary embedding, Eq. 3 bias per token and head, cast), the read of
// cached values, and causal grouped-query attention of new tokens over the
// cache.
//
// Keys lie in a page as rows [token][d_head], values as blocks of 16 tokens
// [d_head][16], so that both products of the attention read what they contract
// over contiguously: keys over d_head, values over tokens.  A page number is
// checked before it is used, so no contents of the page table lead outside the
// cache.
#include "fp8lin_glue.h"

using namespace fp8lin;

namespace {

constexpr int kT = 256;       // threads of every kernel here
constexpr int kBlk = 16;      // tokens of a value block
constexpr int kBf16 = LLAMA_CACHE_BF16;

template <int FMT> constexpr int kEsz = FMT == kBf16 ? 2 : 1;

// ------------------------------------------------------------- sequences
// Largest s < n with f(s) <= x (0 if there is none), f nondecreasing, by one
// wave: each step tests 64 points, so up to 64 sequences take one load.
template <typename F>
__device__ __forceinline__ int wave_search(int n, int64_t x, F f) {
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int i = lane * step;
        const bool le = i < n && f(lo + i) <= x;
        const int cnt = __popcll(__ballot(le));
        const int at = cnt > 0 ? (cnt - 1) * step : 0;
        lo += at;
        n = min(step, n - at);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Rows and positions of sequence s: rows r0 .. r0 + n - 1 of the call are at
// positions p0 .. p0 + n - 1; len keys are present at most.
struct Seq {
    int64_t r0;
    int n, p0, len;
};
__device__ __forceinline__ int64_t row_at(const CacheView& c, int s) {  // cu_rows[s], within the call's rows
    const int64_t v = c.cu[s];
    return v < 0 ? 0 : v > c.rows ? c.rows : v;
}
__device__ __forceinline__ Seq seq_of(const CacheView& c, int s) {
    Seq q;
    q.r0 = row_at(c, s);
    const int64_t r1 = row_at(c, s + 1);
    q.n = r1 > q.r0 ? (int)(r1 - q.r0) : 0;
    const int64_t cap = (int64_t)c.max_pages << c.page_shift;
    const int64_t kv = c.kv_len[s];
    // beyond 2^30 every position is absent, whatever it is
    const int64_t p0 = kv - q.n, lim = (int64_t)1 << 30;
    q.p0 = (int)(p0 < -lim ? -lim : p0 > lim ? lim : p0);
    q.len = (int)(kv < 0 ? 0 : kv < cap ? kv : cap);
    return q;
}
// Page of position p of sequence s, or -1 if it is absent.
__device__ __forceinline__ int page_of(const CacheView& c, int s, int p) {
    const int i = p >> c.page_shift;
    if (p < 0 || i >= c.max_pages) return -1;
    const int g = c.pages[(int64_t)s * c.ld_pages + i];
    return g >= 0 && g < c.n_pages ? g : -1;
}
// Slot (counted over all pages and heads) of position p in page g, head hk:
// times d_head, the element offset of its key row, and for p a multiple of 16
// that of its value block; as it is, that of its exponents.
__device__ __forceinline__ int64_t slot_of(const CacheView& c, int g, int hk, int p) {
    return (((int64_t)g * c.nkv + hk) << c.page_shift) + (p & ((1 << c.page_shift) - 1));
}

// Blocks of 16 consecutive positions (aligned) that sequences touch, one slot
// number each: sequence s owns the slots from cu_rows[s] / 16 + 2 s on, of
// which a sequence of n rows has at least n / 16 + 2 (rounded down), and it touches at
// most (n + 14) / 16 + 1 (rounded down), which is no more.
int64_t block_slots(int64_t rows, int n_seqs) { return rows / kBlk + 2 * (int64_t)n_seqs; }

struct Block {
    int s;       // sequence
    Seq q;
    int b0;      // first position (a multiple of 16; may be negative)
    int t0, t1;  // tokens t0 <= t < t1 of the block are rows of the call
    int64_t row; // row of token t: row + t
};
__device__ __forceinline__ bool block_of(const CacheView& c, int64_t slot, Block* b) {
    b->s = wave_search(c.n_seqs, slot, [&](int s) { return row_at(c, s) / kBlk + 2 * (int64_t)s; });
    b->q = seq_of(c, b->s);
    const int j = (int)(slot - (b->q.r0 / kBlk + 2 * (int64_t)b->s));
    const int first = (b->q.p0 >> 4) << 4;  // rounded down, negatives too
    b->b0 = first + kBlk * j;
    b->t0 = max(b->q.p0 - b->b0, 0);
    b->t1 = min(b->q.p0 + b->q.n - b->b0, kBlk);
    b->row = b->q.r0 + (b->b0 - b->q.p0);
    return b->t0 < b->t1;
}

// ------------------------------------------------------------- append
// Exponent byte of the rows' largest magnitude pattern, and the bias itself.
template <int FMT>
__device__ __forceinline__ int row_bias(uint32_t mag) {
    uint32_t fl;
    return min(bias_of<FMT>(mag, 0, &fl), 126);
}

// Four fp32 values -> four codes with bias b.
template <int FMT>
__device__ __forceinline__ uint32_t codes4(const float* f, int b) {
    const uint4 v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    uint32_t w = cast4_f32<FMT>(v, b);
    const uint32_t hs[4] = {f32_key(v.x), f32_key(v.y), f32_key(v.z), f32_key(v.w)};
    const uint32_t top = max(max(hs[0] & 0x7FFFu, hs[1] & 0x7FFFu), max(hs[2] & 0x7FFFu, hs[3] & 0x7FFFu));
    if (__builtin_expect(top > 0x7F80u, 0)) w = nan_patch<FMT>(w, hs);
    return w;
}

// One workgroup per block of 16 positions and group of heads: each lane holds
// 8 + 8 values of one (token, head), elements 8 j .. of its two halves, which
// are what the rotary embedding pairs.  Workgroups below gqk take query and key
// heads, the others value heads, which they transpose through LDS.
template <int FMT, int DH>
__global__ __launch_bounds__(kT) void append_kernel(CacheView c, const uint16_t* __restrict__ qkv, int64_t ld, int nh,
                                                    const float2* __restrict__ table, uint16_t* __restrict__ q,
                                                    int64_t ldq, int gqk) {
    constexpr int kLanes = DH / 16;                // lanes of one (token, head)
    constexpr int kHeads = kT / (kBlk * kLanes);   // heads at a time
    constexpr int kE = FMT == kBf16 ? 1 : FMT;     // a format for the code that bf16 does not run
    __shared__ __attribute__((aligned(16))) uint8_t vt[kHeads * DH * kBlk * kEsz<FMT>];
    Block b;
    if (!block_of(c, blockIdx.x, &b)) return;
    const int tid = threadIdx.x, j = tid % kLanes, t = (tid / kLanes) % kBlk, hs = tid / (kLanes * kBlk);
    const int pos = b.b0 + t;
    const bool live = t >= b.t0 && t < b.t1;
    const int page = b.b0 < 0 ? -1 : page_of(c, b.s, b.b0);  // one page: page sizes are multiples of 16
    const uint16_t* xr = qkv + (b.row + t) * ld;
    if ((int)blockIdx.y < gqk) {
        const int h = blockIdx.y * kHeads + hs;
        if (!live || h >= nh + c.nkv) return;  // whole groups of kLanes lanes leave together
        if (h < nh && !q) return;
        const uint16_t* x = xr + (int64_t)h * DH + 8 * j;
        const uint4 lo = ld16(x), hi = ld16(x + DH / 2);
        const uint32_t aw[4] = {lo.x, lo.y, lo.z, lo.w}, bw[4] = {hi.x, hi.y, hi.z, hi.w};
        float f0[8], f1[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f0[2 * k] = lo_f(aw[k]);
            f0[2 * k + 1] = hi_f(aw[k]);
            f1[2 * k] = lo_f(bw[k]);
            f1[2 * k + 1] = hi_f(bw[k]);
        }
        if (table && page >= 0) {  // absent positions are not in the table, and not stored
            const float2* cs = table + (int64_t)pos * (DH / 2) + 8 * j;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float2 e = cs[k];
                // In fp64, where the products are exact: a difference that
                // cancels lands on the right side of the border between two
                // codes.  The kernel waits for memory, not for this.
                const double a = f0[k], d = f1[k];
                f0[k] = (float)(a * e.x - d * e.y);
                f1[k] = (float)(d * e.x + a * e.y);
            }
        }
        if (h < nh) {
            uint16_t* o = q + (b.row + t) * ldq + (int64_t)h * DH + 8 * j;
            uint4 u = make_uint4(0u, 0u, 0u, 0u), w = u;
            if (page >= 0) {
                u = make_uint4(pack_bf16x2(f0[0], f0[1]), pack_bf16x2(f0[2], f0[3]), pack_bf16x2(f0[4], f0[5]), pack_bf16x2(f0[6], f0[7]));
                w = make_uint4(pack_bf16x2(f1[0], f1[1]), pack_bf16x2(f1[2], f1[3]), pack_bf16x2(f1[4], f1[5]), pack_bf16x2(f1[6], f1[7]));
            }
            st16(o, u);
            st16(o + DH / 2, w);
            return;
        }
        if (page < 0) return;
        const int64_t slot = slot_of(c, page, h - nh, pos);
        if (FMT == kBf16) {
            uint16_t* o = (uint16_t*)c.k + slot * DH + 8 * j;
            st16(o, make_uint4(pack_bf16x2(f0[0], f0[1]), pack_bf16x2(f0[2], f0[3]), pack_bf16x2(f0[4], f0[5]), pack_bf16x2(f0[6], f0[7])));
            st16(o + DH / 2, make_uint4(pack_bf16x2(f1[0], f1[1]), pack_bf16x2(f1[2], f1[3]), pack_bf16x2(f1[4], f1[5]), pack_bf16x2(f1[6], f1[7])));
            return;
        }
        uint32_t mag = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) mag = max(mag, max(__float_as_uint(f0[k]) & 0x7FFFFFFFu, __float_as_uint(f1[k]) & 0x7FFFFFFFu));
#pragma unroll
        for (int off = 1; off < kLanes; off <<= 1) mag = max(mag, (uint32_t)__shfl_xor((int)mag, off, 64));
        const int bias = row_bias<kE>(mag);
        uint8_t* o = c.k + slot * DH + 8 * j;
        *(uint2*)o = make_uint2(codes4<kE>(f0, bias), codes4<kE>(f0 + 4, bias));
        *(uint2*)(o + DH / 2) = make_uint2(codes4<kE>(f1, bias), codes4<kE>(f1 + 4, bias));
        if (j == 0) c.ke[slot] = (uint8_t)(127 - bias);
        return;
    }
    // value heads: codes of the 16 tokens into LDS as [head][d][16], then out
    // in the same order
    if (page < 0) return;
    const int hv0 = (blockIdx.y - gqk) * kHeads, hv = hv0 + hs;
    if (live && hv < c.nkv) {
        const uint16_t* x = xr + (int64_t)(nh + c.nkv + hv) * DH + 16 * j;
        const uint4 lo = ld16(x), hi = ld16(x + 8);
        const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        uint8_t* row = vt + (hs * DH + 16 * j) * kBlk * kEsz<FMT>;
        if (FMT == kBf16) {
#pragma unroll
            for (int k = 0; k < 16; ++k) ((uint16_t*)row)[k * kBlk + t] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
        } else {
            float f[16];
            uint32_t mag = 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                f[k] = k & 1 ? hi_f(w[k >> 1]) : lo_f(w[k >> 1]);
                mag = max(mag, __float_as_uint(f[k]) & 0x7FFFFFFFu);
            }
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) mag = max(mag, (uint32_t)__shfl_xor((int)mag, off, 64));
            const int bias = row_bias<kE>(mag);
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
                const uint32_t cw = codes4<kE>(f + k, bias);
#pragma unroll
                for (int e = 0; e < 4; ++e) row[(k + e) * kBlk + t] = (uint8_t)(cw >> (8 * e));
            }
            if (j == 0) c.ve[slot_of(c, page, hv, pos)] = (uint8_t)(127 - bias);
        }
    }
    __syncthreads();
    const int d = tid % DH, hd = tid / DH;  // one row of 16 tokens per thread: kHeads * DH = kT
    if (hv0 + hd >= c.nkv) return;
    const uint8_t* src = vt + tid * kBlk * kEsz<FMT>;
    uint8_t* dst = c.v + (slot_of(c, page, hv0 + hd, b.b0) * DH + d * kBlk) * kEsz<FMT>;
    if (b.t0 == 0 && b.t1 == kBlk) {
        st16(dst, ld16(src));
        if (FMT == kBf16) st16(dst + 16, ld16(src + 16));
    } else {  // the other tokens of the block keep their values
        for (int k = b.t0; k < b.t1; ++k) {
            if (FMT == kBf16) ((uint16_t*)dst)[k] = ((const uint16_t*)src)[k];
            else dst[k] = src[k];
        }
    }
}

// ------------------------------------------------------------- decode of codes
// Codes 0..3 of a word -> fp32 (exact).
template <int FMT, int I>
__device__ __forceinline__ float decode(uint32_t w) {
    return FMT == FP8_E5M2 ? __builtin_amdgcn_cvt_f32_bf8((int)w, I) : __builtin_amdgcn_cvt_f32_fp8((int)w, I);
}
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float* f) {
    f[0] = decode<FMT, 0>(w);
    f[1] = decode<FMT, 1>(w);
    f[2] = decode<FMT, 2>(w);
    f[3] = decode<FMT, 3>(w);
}
// 2^(e - 127) of an exponent byte (0: 2^-127, 255: NaN).
__device__ __forceinline__ float unscale_of(uint32_t e) { return ldexpf(e == 255u ? __builtin_nanf("") : 1.0f, (int)e - 127); }

// ------------------------------------------------------------- read
// The same blocks and head groups; blockIdx.y below gk reads keys (each lane 16
// values of one token), the others values through the transpose.
template <int FMT, int DH>
__global__ __launch_bounds__(kT) void read_kernel(CacheView c, uint16_t* __restrict__ ko, int64_t ldk,
                                                  uint16_t* __restrict__ vo, int64_t ldv, int gk) {
    constexpr int kLanes = DH / 16, kHeads = kT / (kBlk * kLanes);
    constexpr int kE = FMT == kBf16 ? 1 : FMT;
    __shared__ __attribute__((aligned(16))) uint8_t vt[kHeads * DH * kBlk * kEsz<FMT>];
    Block b;
    if (!block_of(c, blockIdx.x, &b)) return;
    const bool keys = (int)blockIdx.y < gk;
    const int h0 = (keys ? blockIdx.y : blockIdx.y - gk) * kHeads;
    const int tid = threadIdx.x, j = tid % kLanes, t = (tid / kLanes) % kBlk, hs = tid / (kLanes * kBlk), h = h0 + hs;
    const int page = b.b0 < 0 ? -1 : page_of(c, b.s, b.b0);
    const bool live = t >= b.t0 && t < b.t1 && h < c.nkv;
    if (!keys && page >= 0) {
        const int d = tid % DH, hd = tid / DH;
        if (h0 + hd < c.nkv) {
            const uint8_t* src = c.v + (slot_of(c, page, h0 + hd, b.b0) * DH + d * kBlk) * kEsz<FMT>;
            uint8_t* dst = vt + tid * kBlk * kEsz<FMT>;
            st16(dst, ld16(src));
            if (FMT == kBf16) st16(dst + 16, ld16(src + 16));
        }
    }
    __syncthreads();
    if (!live) return;
    uint16_t* o = (keys ? ko + (b.row + t) * ldk : vo + (b.row + t) * ldv) + (int64_t)h * DH + 16 * j;
    uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    if (page >= 0) {
        const int64_t slot = slot_of(c, page, h, b.b0 + t);
        const uint8_t* row = vt + (hs * DH + 16 * j) * kBlk * kEsz<FMT>;
        if (FMT == kBf16) {
            if (keys) {
                const uint16_t* p = (const uint16_t*)c.k + slot * DH + 16 * j;
                const uint4 a = ld16(p), e = ld16(p + 8);
                w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
                w[4] = e.x; w[5] = e.y; w[6] = e.z; w[7] = e.w;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    w[k] = ((const uint16_t*)row)[2 * k * kBlk + t] | ((uint32_t)((const uint16_t*)row)[(2 * k + 1) * kBlk + t] << 16);
            }
        } else {
            uint32_t cw[4];
            if (keys) {
                const uint4 a = ld16(c.k + slot * DH + 16 * j);
                cw[0] = a.x; cw[1] = a.y; cw[2] = a.z; cw[3] = a.w;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    cw[k] = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) cw[k] |= (uint32_t)row[(4 * k + e) * kBlk + t] << (8 * e);
                }
            }
            const float sc = unscale_of(keys ? c.ke[slot] : c.ve[slot]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float f[4];
                decode4<kE>(cw[k], f);
                w[2 * k] = pack_bf16x2(f[0] * sc, f[1] * sc);
                w[2 * k + 1] = pack_bf16x2(f[2] * sc, f[3] * sc);
            }
        }
    }
    st16(o, make_uint4(w[0], w[1], w[2], w[3]));
    st16(o + 8, make_uint4(w[4], w[5], w[6], w[7]));
}

// ------------------------------------------------------------- attention
// One wave per (row, head): keys in tiles of 64, one per lane; running maximum
// and sum of the softmax; each lane then sums two (or one) dimensions of the
// values.
template <int FMT, int DH, bool QUANT, int QF>
__global__ __launch_bounds__(kT) void attn_kernel(CacheView c, const uint16_t* __restrict__ q, int64_t ldq, int nh,
                                                  int64_t max_rows, int64_t window, uint16_t* __restrict__ o,
                                                  int64_t ldo, const int32_t* __restrict__ pred,
                                                  int32_t* __restrict__ used, uint32_t* __restrict__ parts,
                                                  uint8_t* __restrict__ q8, int64_t ldq8) {
    constexpr int kE = FMT == kBf16 ? 1 : FMT, kPer = DH / 64;
    __shared__ float qs[kT / 64][DH];
    __shared__ uint32_t redm[kT / 64];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int bq = QUANT ? fused_bias(pred, used) : 0;
    const int64_t item = (int64_t)blockIdx.x * (kT / 64) + w;
    const int64_t r = item / nh;
    const int h = (int)(item % nh), hk = h / (nh / c.nkv);
    const int s = wave_search(c.n_seqs, r, [&](int i) { return row_at(c, i); });
    const Seq sq = seq_of(c, s);
    const bool live = r < c.rows && r >= sq.r0 && r < sq.r0 + sq.n && r - sq.r0 < max_rows;
    uint32_t mag = 0;
    if (live) {
        for (int i = lane; i < DH; i += 64) qs[w][i] = lo_f(q[r * ldq + (int64_t)h * DH + i]);
    }
    __syncthreads();
    if (live) {
        const int64_t p = (int64_t)sq.p0 + (r - sq.r0);
        const int64_t kend = min(p + 1, (int64_t)sq.len);
        const int64_t klo = window > 0 ? max(p - window + 1, (int64_t)0) : 0;
        const float scale = 1.4426950408889634f / sqrtf((float)DH);
        float m = -INFINITY, l = 0.0f, acc[kPer];
        for (int i = 0; i < kPer; ++i) acc[i] = 0.0f;
        for (int64_t k0 = klo & ~(int64_t)63; k0 < kend; k0 += 64) {
            const int64_t key = k0 + lane;
            const int page = key >= klo && key < kend ? page_of(c, s, (int)key) : -1;
            const int64_t slot = page >= 0 ? slot_of(c, page, hk, (int)key) : 0;
            float sc = 0.0f, vs = 1.0f;
            if (page >= 0) {
                for (int d = 0; d < DH; d += 4) {
                    float f[4];
                    if (FMT == kBf16) {
                        const uint2 u = *(const uint2*)((const uint16_t*)c.k + slot * DH + d);
                        f[0] = lo_f(u.x); f[1] = hi_f(u.x); f[2] = lo_f(u.y); f[3] = hi_f(u.y);
                    } else {
                        decode4<kE>(*(const uint32_t*)(c.k + slot * DH + d), f);
                    }
                    for (int e = 0; e < 4; ++e) sc += f[e] * qs[w][d + e];
                }
                if (FMT != kBf16) {
                    sc *= unscale_of(c.ke[slot]);
                    vs = unscale_of(c.ve[slot]);
                }
            }
            const float x = page >= 0 ? sc * scale : -INFINITY;
            float mx = x;
            for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
            const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.0f : mn;
            const float alpha = exp2f(m - ref);
            const float pr = page >= 0 ? exp2f(x - ref) : 0.0f;
            l = l * alpha + wave_sum(pr);
            m = mn;
            const float pv = pr * vs;
            for (int i = 0; i < kPer; ++i) acc[i] *= alpha;
            for (int k = 0; k < 64; ++k) {
                const int pg = __shfl(page, k, 64);
                if (pg < 0) continue;
                const int64_t sl = slot_of(c, pg, hk, (int)(k0 + k));
                const float pk = __shfl(pv, k, 64);
                const int64_t vb = (sl & ~(int64_t)15) * DH + (sl & 15);
                for (int i = 0; i < kPer; ++i) {
                    const int64_t at = vb + (int64_t)(lane * kPer + i) * kBlk;
                    const float v = FMT == kBf16 ? lo_f(((const uint16_t*)c.v)[at]) : decode<kE, 0>(c.v[at]);
                    acc[i] += pk * v;
                }
            }
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        for (int i = 0; i < kPer; ++i) {
            const uint32_t u = pack_bf16x2(acc[i] * inv, 0.0f) & 0xFFFFu;
            const int64_t col = (int64_t)h * DH + lane * kPer + i;
            o[r * ldo + col] = (uint16_t)u;
            if (QUANT) {
                mag = max(mag, u & 0x7FFFu);
                if (pred) q8[r * ldq8 + col] = (uint8_t)codes8<QF>(make_uint4(u, 0u, 0u, 0u), bq).x;
            }
        }
    }
    if (QUANT) {
        const uint32_t bm = block_max(mag, redm);
        if (threadIdx.x == 0) parts[blockIdx.x] = bm;
    }
}

// ------------------------------------------------------------- fused quantise
// The exact bias of the output from the workgroups' maxima, and the codes of
// the rows of sequences again where they were cast with another one.
template <int QF>
__global__ __launch_bounds__(kT) void quant_finish_kernel(CacheView c, const uint16_t* __restrict__ o, int64_t cols,
                                                          int64_t ldo, int64_t max_rows, int32_t margin,
                                                          const uint32_t* __restrict__ ws, int nparts,
                                                          int32_t* __restrict__ bias, uint32_t* __restrict__ amax_bits,
                                                          uint32_t* __restrict__ flags, uint8_t* __restrict__ q8,
                                                          int64_t ldq8) {
    __shared__ uint32_t red[kT / 64];
    __shared__ uint32_t amax_s;
    const uint32_t m = block_max(strided_max<kT>(ws + 1, nparts), red);
    if (threadIdx.x == 0) amax_s = m;
    __syncthreads();
    const uint32_t a32 = canon_amax(amax_s << 16);
    uint32_t fl;
    const int32_t bx = bias_of<QF>(a32, margin, &fl);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *bias = bx;
        if (amax_bits) *amax_bits = a32;
        if (flags) *flags = fl;
    }
    const int b = clamp_bias(bx);
    if ((int32_t)ws[0] == b) return;
    for (int64_t r = blockIdx.x; r < c.rows; r += gridDim.x) {
        const int s = wave_search(c.n_seqs, r, [&](int i) { return row_at(c, i); });
        const Seq sq = seq_of(c, s);
        if (r < sq.r0 || r >= sq.r0 + sq.n || r - sq.r0 >= max_rows) continue;
        for (int64_t col = 8 * threadIdx.x; col < cols; col += 8 * kT)
            *(uint2*)(q8 + r * ldq8 + col) = codes8<QF>(ld16(o + r * ldo + col), b);
    }
}

// ------------------------------------------------------------- host side
template <typename Fn>
void with_cache(int fmt, int d_head, Fn&& fn) {
    auto go = [&](auto F) {
        if (d_head == 128) fn(F, IC<128>{});
        else fn(F, IC<64>{});
    };
    if (fmt == FP8_E4M3) go(IC<FP8_E4M3>{});
    else if (fmt == FP8_E5M2) go(IC<FP8_E5M2>{});
    else go(IC<kBf16>{});
}

}  // namespace

namespace fp8lin {

int32_t launch_cache_append(const uint16_t* qkv, int64_t ld, int nh, const CacheView& c, int fmt, int d_head,
                            const float* table, uint16_t* q, int64_t ldq, hipStream_t s) {
    const int per = kT / d_head;  // heads of one workgroup
    const int gqk = (nh + c.nkv + per - 1) / per, gv = (c.nkv + per - 1) / per;
    const dim3 grid((unsigned)block_slots(c.rows, c.n_seqs), (unsigned)(gqk + gv));
    with_cache(fmt, d_head, [&](auto F, auto D) {
        hipLaunchKernelGGL((append_kernel<decltype(F)::value, decltype(D)::value>), grid, dim3(kT), 0, s, c, qkv, ld, nh,
                           (const float2*)table, q, ldq, gqk);
    });
    return hip_status();
}

int32_t launch_cache_read(const CacheView& c, int fmt, int d_head, uint16_t* k, int64_t ldk, uint16_t* v, int64_t ldv,
                          hipStream_t s) {
    const int per = kT / d_head, g = (c.nkv + per - 1) / per;
    const dim3 grid((unsigned)block_slots(c.rows, c.n_seqs), (unsigned)((k ? g : 0) + (v ? g : 0)));
    with_cache(fmt, d_head, [&](auto F, auto D) {
        hipLaunchKernelGGL((read_kernel<decltype(F)::value, decltype(D)::value>), grid, dim3(kT), 0, s, c, k, ldk, v, ldv,
                           k ? g : 0);
    });
    return hip_status();
}

CacheAttnPlan cache_attn_plan(int64_t rows, int nh, int nkv, int d_head, int64_t n_seqs, int64_t max_rows,
                              int64_t max_len) {
    CacheAttnPlan p;
    p.parts = (rows * nh + kT / 64 - 1) / (kT / 64);
    p.ws_bytes = (1 + p.parts) * (int64_t)sizeof(uint32_t);
    return p;
}

int32_t launch_cache_attention(const uint16_t* q, int64_t ldq, int nh, const CacheView& c, int fmt, int d_head,
                               int64_t max_rows, int64_t window, uint16_t* o, int64_t ldo, const FusedQuant* fq,
                               void* ws, hipStream_t s) {
    const bool quant = fq && fq->q;
    const CacheAttnPlan p = cache_attn_plan(c.rows, nh, c.nkv, d_head, c.n_seqs, max_rows,
                                            (int64_t)c.max_pages << c.page_shift);
    uint32_t* words = (uint32_t*)ws;
    with_cache(fmt, d_head, [&](auto F, auto D) {
        with_fmt(quant ? fq->fmt : FP8_E4M3, [&](auto QF) {
            constexpr int kF = decltype(F)::value, kD = decltype(D)::value, kQ = decltype(QF)::value;
            if (quant)
                hipLaunchKernelGGL((attn_kernel<kF, kD, true, kQ>), dim3((unsigned)p.parts), dim3(kT), 0, s, c, q, ldq,
                                   nh, max_rows, window, o, ldo, fq->pred, (int32_t*)words, words + 1, fq->q, fq->ldq);
            else
                hipLaunchKernelGGL((attn_kernel<kF, kD, false, kQ>), dim3((unsigned)p.parts), dim3(kT), 0, s, c, q, ldq,
                                   nh, max_rows, window, o, ldo, nullptr, nullptr, nullptr, nullptr, (int64_t)0);
        });
    });
    int32_t st = hip_status();
    if (st == FP8_OK && quant) {
        const int64_t cols = (int64_t)nh * d_head;
        with_fmt(fq->fmt, [&](auto QF) {
            hipLaunchKernelGGL((quant_finish_kernel<decltype(QF)::value>), dim3((unsigned)(c.rows < 512 ? c.rows : 512)),
                               dim3(kT), 0, s, c, o, cols, ldo, max_rows, fq->margin, words, (int)p.parts, fq->bias,
                               fq->amax_bits, fq->flags, fq->q, fq->ldq);
        });
        st = hip_status();
    }
    return st;
}

}  // namespace fp8lin
