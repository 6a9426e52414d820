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
// Workgroups of append and read that heads are grouped for: 4096 (64 single tokens
// of 80 heads 5.9 us, read of 2464 tokens of 2 x 32 heads 15.0; with 2048: 5.3 and 17.1, with
// 8192: 8.3 and 14.3).
constexpr int kBlockWgs = 4096;

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

// Place of row r (of 16 tokens) in the LDS copy of a value block: a row's space is
// left out after every 16, so that lanes on rows 16 apart are on other banks.
__host__ __device__ constexpr int vt_row(int r) { return r + (r >> 4); }

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

// A workgroup takes a block of 16 positions and a group of heads, as many (token,
// head) at a time as it has lanes for (DH / 16 lanes each, 16 values a lane: all
// tokens of two heads of 128 for a whole block, 32 heads for a single token), with
// the next ones' loads under way.  Bound by memory once the
// first loads (sequence, lengths, page, table) are there, which the many
// workgroups hide from each other.  Measured: 2048 tokens of 80 heads in 17.9 us
// (80 MB at 4.5 TB/s), 64 single tokens in 5.9 us, one in 3.8 us.
template <int FMT, int DH>
struct Append {
    static constexpr int kLanes = DH / 16;                // lanes of one (token, head)
    static constexpr int kUnits = kT / kLanes;            // (token, head) at a time
    static constexpr int kE = FMT == kBf16 ? 1 : FMT;     // a format for the code that bf16 does not run

    // Largest magnitude pattern over the lanes of a (token, head), as a bias.
    static __device__ __forceinline__ int bias(uint32_t mag) {
#pragma unroll
        for (int off = 1; off < kLanes; off <<= 1) mag = max(mag, (uint32_t)__shfl_xor((int)mag, off, 64));
        return row_bias<kE>(mag);
    }
};

__device__ __forceinline__ void halves(uint4 v, float* f) {  // eight bf16 -> fp32
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f[2 * k] = lo_f(w[k]);
        f[2 * k + 1] = hi_f(w[k]);
    }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ uint32_t mag_f(const float* f, int n, uint32_t m) {
#pragma unroll
    for (int k = 0; k < n; ++k) m = max(m, __float_as_uint(f[k]) & 0x7FFFFFFFu);
    return m;
}

// Groups below gqk: heads_qk query and key heads each, others: heads_v value heads.
// q may be qkv's query columns: a lane writes there what it has read before.
template <int FMT, int DH>
__global__ __launch_bounds__(kT) void append_kernel(CacheView c, const uint16_t* qkv, int64_t ld, int nh,
                                                    const float2* __restrict__ table, uint16_t* q, int64_t ldq, int gqk,
                                                    int heads_qk, int heads_v) {
    using A = Append<FMT, DH>;
    constexpr int kLanes = A::kLanes, kE = A::kE, kPair = A::kUnits / kBlk;  // heads of a whole block at a time
    __shared__ __attribute__((aligned(16))) uint8_t vt[vt_row(kPair * DH) * kBlk * kEsz<FMT>];
    Block b;
    if (!block_of(c, blockIdx.x, &b)) return;
    const int tid = threadIdx.x, j = tid % kLanes, unit = tid / kLanes, nt = b.t1 - b.t0;
    const int per = A::kUnits / nt;  // heads at a time
    const int hs = unit / nt, t = b.t0 + unit % nt, pos = b.b0 + t;
    const int page = b.b0 < 0 ? -1 : page_of(c, b.s, b.b0);  // one page: page sizes are multiples of 16
    const int64_t row = b.row + t;
    if ((int)blockIdx.y < gqk) {
        const int first = blockIdx.y * heads_qk + (q ? 0 : nh), end = min(first + heads_qk, nh + c.nkv);
        if (hs >= per) return;  // lanes of one (token, head) stay together
        const uint16_t* x = qkv + row * ld + 8 * j;  // elements 8 j .. of the two halves, which the rotation pairs
        int h = first + hs;
        if (h >= end) return;
        uint4 lo = ld16(x + (int64_t)h * DH), hi = ld16(x + (int64_t)h * DH + DH / 2);
        float2 cs[8];
        const bool turn = table && page >= 0;  // absent positions are not in the table, and not stored
        if (turn) {
            const float4* tp = (const float4*)(table + (int64_t)pos * (DH / 2) + 8 * j);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 e = tp[k];
                cs[2 * k] = make_float2(e.x, e.y);
                cs[2 * k + 1] = make_float2(e.z, e.w);
            }
        }
        for (; h < end; h += per) {
            float f0[8], f1[8];
            halves(lo, f0);
            halves(hi, f1);
            if (h + per < end) {
                lo = ld16(x + (int64_t)(h + per) * DH);
                hi = ld16(x + (int64_t)(h + per) * DH + DH / 2);
            }
            if (turn) {
                // In fp64, where the products are exact: a difference that cancels
                // lands on the right side of the border between two codes.
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const double u = f0[k], v = f1[k], co = cs[k].x, si = cs[k].y;
                    f0[k] = (float)(u * co - v * si);
                    f1[k] = (float)(v * co + u * si);
                }
            }
            if (h < nh) {
                uint16_t* o = q + row * ldq + (int64_t)h * DH + 8 * j;
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                st16(o, page >= 0 ? pack8(f0) : zero);
                st16(o + DH / 2, page >= 0 ? pack8(f1) : zero);
                continue;
            }
            if (page < 0) continue;
            const int64_t slot = slot_of(c, page, h - nh, pos);
            if (FMT == kBf16) {
                uint16_t* o = (uint16_t*)c.k + slot * DH + 8 * j;
                st16(o, pack8(f0));
                st16(o + DH / 2, pack8(f1));
                continue;
            }
            const int bias = A::bias(mag_f(f1, 8, mag_f(f0, 8, 0u)));
            uint8_t* o = c.k + slot * DH + 8 * j;
            *(uint2*)o = make_uint2(codes4<kE>(f0, bias), codes4<kE>(f0 + 4, bias));
            *(uint2*)(o + DH / 2) = make_uint2(codes4<kE>(f1, bias), codes4<kE>(f1 + 4, bias));
            if (j == 0) c.ke[slot] = (uint8_t)(127 - bias);
        }
        return;
    }
    // Value heads, 16 consecutive values a lane.  A whole block is transposed
    // through LDS and leaves as 16-byte (bf16: 32-byte) rows of a dimension; of a
    // part of a block, each value goes to its place, and the other tokens keep theirs.
    if (page < 0) return;
    const int first = (blockIdx.y - gqk) * heads_v, end = min(first + heads_v, c.nkv);
    const uint16_t* x = qkv + row * ld + (int64_t)(nh + c.nkv) * DH + 16 * j;
    const bool whole = nt == kBlk;
    for (int h0 = first; h0 < end; h0 += per) {
        const int h = h0 + hs;
        const bool live = hs < per && h < end;
        if (live) {
            const uint4 lo = ld16(x + (int64_t)h * DH), hi = ld16(x + (int64_t)h * DH + 8);
            const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            const int64_t slot = slot_of(c, page, h, pos);
            // the lane's first dimension of this token, in LDS or in the cache
            uint8_t* dst = whole ? vt + (vt_row(hs * DH + 16 * j) * kBlk + t) * kEsz<FMT>
                                 : c.v + ((slot - t) * DH + 16 * j * kBlk + t) * kEsz<FMT>;
            if (FMT == kBf16) {
#pragma unroll
                for (int k = 0; k < 16; ++k) ((uint16_t*)dst)[k * kBlk] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
            } else {
                float f[16];
                halves(lo, f);
                halves(hi, f + 8);
                const int bias = A::bias(mag_f(f, 16, 0u));
#pragma unroll
                for (int k = 0; k < 16; k += 4) {
                    const uint32_t cw = codes4<kE>(f + k, bias);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dst[(k + e) * kBlk] = (uint8_t)(cw >> (8 * e));
                }
                if (j == 0) c.ve[slot] = (uint8_t)(127 - bias);
            }
        }
        if (whole) {
            __syncthreads();
            const int d = tid % DH, hd = h0 + tid / DH;  // one row of 16 tokens per thread
            if (hd < end) {
                const uint8_t* src = vt + vt_row(tid) * kBlk * kEsz<FMT>;
                uint8_t* dst = c.v + (slot_of(c, page, hd, b.b0) * DH + d * kBlk) * kEsz<FMT>;
                st16(dst, ld16(src));
                if (FMT == kBf16) st16(dst + 16, ld16(src + 16));
            }
            __syncthreads();
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
// 2^(e - 127) of an exponent byte (0: 2^-127; 255 counts as 254, so that the weight 0 of
// a token that a row does not see stays 0).
__device__ __forceinline__ float exp_float(uint32_t e) {
    return __uint_as_float(min(max(e << 23, 0x00400000u), 0x7F000000u));
}

// ------------------------------------------------------------- read
// The same blocks; groups of `heads` heads, keys below gk, then values.  A
// workgroup reads whole blocks of as many heads as it has lanes for, the next
// ones' loads under way: keys as they lie, values through a transpose in LDS.
template <int FMT, int DH>
__global__ __launch_bounds__(kT) void read_kernel(CacheView c, uint16_t* __restrict__ ko, int64_t ldk,
                                                  uint16_t* __restrict__ vo, int64_t ldv, int gk, int heads) {
    constexpr int kLanes = DH / 16, kPair = kT / (kBlk * kLanes);
    constexpr int kE = FMT == kBf16 ? 1 : FMT, kV = kEsz<FMT>;  // vectors of a lane
    __shared__ __attribute__((aligned(16))) uint8_t vt[vt_row(kPair * DH) * kBlk * kEsz<FMT>];
    Block b;
    if (!block_of(c, blockIdx.x, &b)) return;
    const bool keys = (int)blockIdx.y < gk;
    const int first = (keys ? blockIdx.y : blockIdx.y - gk) * heads, end = min(first + heads, c.nkv);
    const int tid = threadIdx.x, j = tid % kLanes, t = (tid / kLanes) % kBlk, hs = tid / (kLanes * kBlk);
    const int page = b.b0 < 0 ? -1 : page_of(c, b.s, b.b0);
    const bool live = t >= b.t0 && t < b.t1;
    uint16_t* out = (keys ? ko + (b.row + t) * ldk : vo + (b.row + t) * ldv) + 16 * j;
    if (page < 0) {  // absent: zeros
        for (int h = first + hs; h < end; h += kPair)
            if (live) {
                st16(out + (int64_t)h * DH, make_uint4(0u, 0u, 0u, 0u));
                st16(out + (int64_t)h * DH + 8, make_uint4(0u, 0u, 0u, 0u));
            }
        return;
    }
    // what this lane loads of a block: 16 dimensions of its token's key, or the 16
    // tokens of dimension tid % DH of head tid / DH
    const int ls = keys ? hs : tid / DH;
    const int at = keys ? t * DH + 16 * j : (tid % DH) * kBlk;
    const uint8_t* src = (keys ? c.k : c.v) + at * kEsz<FMT>;
    const uint8_t* exps = keys ? c.ke : c.ve;
    auto load = [&](int h0, uint4 (&v)[kV], uint32_t& e) {  // a head past the last one: the last one again
        const int64_t slot = slot_of(c, page, min(h0 + ls, end - 1), b.b0);
#pragma unroll
        for (int k = 0; k < kV; ++k) v[k] = ld16(src + slot * DH * kEsz<FMT> + 16 * k);
        if (FMT != kBf16) e = exps[slot_of(c, page, min(h0 + hs, end - 1), b.b0 + t)];
    };
    uint4 v[kV];
    uint32_t e = 0;
    load(first, v, e);
    for (int h0 = first; h0 < end; h0 += kPair) {
        uint4 x[kV];
        const uint32_t ex = e;
#pragma unroll
        for (int k = 0; k < kV; ++k) x[k] = v[k];
        if (h0 + kPair < end) load(h0 + kPair, v, e);
        if (!keys) {
#pragma unroll
            for (int k = 0; k < kV; ++k) st16(vt + vt_row(tid) * kBlk * kEsz<FMT> + 16 * k, x[k]);
            __syncthreads();
            const uint8_t* col = vt + (vt_row(hs * DH + 16 * j) * kBlk + t) * kEsz<FMT>;
            uint32_t w[4 * kV];
            if (FMT == kBf16) {
#pragma unroll
                for (int k = 0; k < 4 * kV; ++k)
                    w[k] = ((const uint16_t*)col)[2 * k * kBlk] | ((uint32_t)((const uint16_t*)col)[(2 * k + 1) * kBlk] << 16);
            } else {
#pragma unroll
                for (int k = 0; k < 4 * kV; ++k)
                    w[k] = col[4 * k * kBlk] | ((uint32_t)col[(4 * k + 1) * kBlk] << 8) |
                           ((uint32_t)col[(4 * k + 2) * kBlk] << 16) | ((uint32_t)col[(4 * k + 3) * kBlk] << 24);
            }
#pragma unroll
            for (int k = 0; k < kV; ++k) x[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
            __syncthreads();
        }
        const int h = h0 + hs;
        if (!live || h >= end) continue;
        uint4 o0, o1;
        if (FMT == kBf16) {
            o0 = x[0];
            o1 = x[kV - 1];
        } else {
            const float sc = exp_float(ex);
            const uint32_t cw[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
            float f[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) decode4<kE>(cw[k], f + 4 * k);
#pragma unroll
            for (int k = 0; k < 16; ++k) f[k] *= sc;
            o0 = pack8(f);
            o1 = pack8(f + 8);
        }
        // streaming stores: 25.0 -> 24.3 us for 16384 tokens of 8 heads
        __builtin_nontemporal_store(u32x4{o0.x, o0.y, o0.z, o0.w}, (u32x4*)(out + (int64_t)h * DH));
        __builtin_nontemporal_store(u32x4{o1.x, o1.y, o1.z, o1.w}, (u32x4*)(out + (int64_t)h * DH + 8));
    }
}

// ------------------------------------------------------------- attention
// A call's rows of one sequence and key/value head form the packed rows m =
// token * group + head of the group: all of them read the same keys.  Two
// kernels, both with the scores transposed (S^T = K . Q^T, then O^T += V^T . P^T),
// so that the probabilities a lane holds are already the operand of the second
// product:
//   few_body   up to 16 packed rows (single tokens): each wave takes tiles of
//                64 keys on its own, keys and values from memory straight into
//                the operand registers; bound by reading the cache;
//   many_body  tiles of 128 packed rows: keys and values through LDS, there in
//                bf16; bound by the matrix cores and the exponentials.
// FP8 codes become bf16 exactly (v_cvt_scalef32_pk_bf16_*).  Both products run
// on the bf16 matrix instructions: those of FP8 operands keep about 14 bits of
// the largest product of a sum (measured: up to 1e-4 of sum |q k| off, against
// 1e-7), which scores do not tolerate.  A key's exponent is applied by that
// conversion; a value's multiplies its probability, whose lanes are along keys.
//
// The key range of a tile of rows can be split over several workgroups, which
// leave (maximum, sum, unnormalised output) in fp32: few_body's are joined by the
// workgroup that ends last, many_body's by many_join_kernel.
typedef float f16_t __attribute__((ext_vector_type(16)));

constexpr int kFew = 16;      // packed rows of few_body
constexpr int kFewW = 4, kFewT = 64 * kFewW;  // its waves and threads
constexpr int kMany = 128;    // packed rows of a workgroup of many_body
constexpr int kTile = 64;     // keys of a tile
// many_body: workgroups that key ranges are cut for (two on a compute unit: 512 tokens
// over 8192 before them, 64 heads in groups of 8, take 201 us with 1024 and 188 with
// 512), and tiles of a range at least.
constexpr int kManyWant = 512, kManyLeast = 8;
constexpr float kLargeScore = 16384.0f;  // many_body: of a maximum times log2(e) / sqrt(d_head), beyond which differences come first
constexpr int kCus = 256;          // compute units
constexpr int kShares = 512;       // workgroups of few_body that run at once
constexpr int kShareLeast = 8;     // tiles of a share at least
constexpr int kFlatTiles = 64;     // of a share, if all sequences were of the longest length, for shares to be worth it
constexpr int kFlatSeqs = 1024;    // sequences that a workgroup counts through
constexpr int kFewPart = 4;        // tiles of a part of an item at least: one step a wave
constexpr int kCounts = LLAMA_CACHE_WS_COUNTS / 4;  // counters at the start of the workspace: items that can be cut

struct AttnArgs {
    CacheView c;
    const uint16_t* q;
    int64_t ldq;
    int nh, grp;
    int max_rows;
    int window;           // 0: none
    int few_on;           // few_body takes the sequences of up to kFew packed rows
    int splits, per;      // many_body's key ranges: how many at most, and tiles of each
    int flat, few_parts;  // few_body: equal shares of all tiles; parts of an item
    int32_t* counts;      // and finished parts of each item
    float c2;             // log2(e) / sqrt(d_head)
    uint16_t* o;
    int64_t ldo;
    // fused quantise (q8 null: none)
    const int32_t* pred;
    int32_t* used;
    uint32_t* parts;      // this launch's
    uint8_t* q8;
    int64_t ldq8;
    int qfmt;
    // partials: output, (maximum, sum); few_body's [share][2][kFew], many_body's
    // [split][row][head]
    float *few_o, *many_o;
    float2 *few_ml, *many_ml;
    int many_wg;          // workgroups of many_body, before those of few_body
};

__device__ __forceinline__ f16_t mfma32(u32x4 a, u32x4 b, f16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}

// Two codes (the low or high half of w) times scale (a power of two) -> two bf16.
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t cvt2b(uint32_t w, float scale) {
    if (FMT == FP8_E5M2) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, HI));
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Eight codes -> eight bf16.
template <int FMT>
__device__ __forceinline__ u32x4 cvt8b(uint32_t w0, uint32_t w1, float scale) {
    return u32x4{cvt2b<FMT, false>(w0, scale), cvt2b<FMT, true>(w0, scale), cvt2b<FMT, false>(w1, scale),
                 cvt2b<FMT, true>(w1, scale)};
}

// Key range of the packed rows m0 .. m1 - 1 of a sequence, as tiles of 64 keys
// from a multiple of 64 on, and the `per` tiles of it that a split takes.
struct Range {
    int start;      // first key of tile 0
    int kend;       // keys below this
    int nt;         // tiles
    int t0, t1;     // tiles of this split
    int live;       // splits that have tiles
    int first, last;  // positions of the first and last row
};
__device__ __forceinline__ Range range_of(const AttnArgs& p, const Seq& sq, int m0, int m1, int split, int per) {
    Range r;
    r.first = sq.p0 + m0 / p.grp;
    r.last = sq.p0 + (m1 - 1) / p.grp;
    r.kend = max(min(r.last + 1, sq.len), 0);
    const int lo = p.window > 0 ? max(r.first - p.window + 1, 0) : 0;
    r.start = lo & ~(kTile - 1);
    const int nt = r.nt = r.kend > r.start ? (r.kend - r.start + kTile - 1) / kTile : 0;
    r.live = (nt + per - 1) / per;
    r.t0 = split * per;
    r.t1 = min(r.t0 + per, nt);
    return r;
}

// Nonfinite values of bf16 pairs: their exponent is all ones.
__device__ __forceinline__ uint32_t nonfinite2(uint32_t w) { return ((w & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u; }

// A value operand that holds infinities or NaN: what a row does not see (weight
// 0) must not reach it, but 0 * NaN would.  So the product takes the finite part,
// and these are indicators (1.0) of +inf or NaN and of -inf or NaN, whose sums over
// the keys that a row sees say whether to add +inf and -inf (both: NaN).
__device__ __forceinline__ void split_nonfinite(u32x4 v, u32x4& up, u32x4& down) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = v[k];
        const uint32_t bad = nonfinite2(w) >> 15;                                     // a 1 in a half that is not finite
        const uint32_t nan = (((w & 0x007F007Fu) + 0x007F007Fu) >> 7) & 0x00010001u;  // whose mantissa is not zero
        const uint32_t neg = (w >> 15) & 0x00010001u;
        up[k] = (bad & (nan | ~neg)) * 0x3F80u;
        down[k] = (bad & (nan | neg)) * 0x3F80u;
    }
}
// 1.0 for each of eight keys whose bit is set.
__device__ __forceinline__ u32x4 ones_where(uint32_t bits) {
    u32x4 m;
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = ((bits >> (2 * k)) & 1u) * 0x3F80u + ((bits >> (2 * k + 1)) & 1u) * 0x3F800000u;
    return m;
}
__device__ __forceinline__ float add_nonfinite(float o, float up, float down) {
    if (up > 0.0f) o += INFINITY;
    if (down > 0.0f) o -= INFINITY;
    return o;
}

// Masks that keep the first n tokens of W words of PER tokens each.
template <int PER, int W>
__device__ __forceinline__ void token_masks(int n, uint32_t (&mk)[W]) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const int bits = max(min(n - PER * k, PER), 0) * (32 / PER);
        mk[k] = (uint32_t)((1ull << bits) - 1);
    }
}

// Eight output values (bf16) of a row: stored, and cast for the fused quantise.
__device__ __forceinline__ uint32_t put8(const AttnArgs& p, bool cast, int bq, int64_t row, int64_t col, uint4 v) {
    st16(p.o + row * p.ldo + col, v);
    if (!p.q8) return 0u;
    if (cast) {
        uint2 u;
        switch (p.qfmt) {
            case FP8_E4M3: u = codes8<FP8_E4M3>(v, bq); break;
            case FP8_E5M2: u = codes8<FP8_E5M2>(v, bq); break;
            case FP8_E4_A: u = codes8<FP8_E4_A>(v, bq); break;
            default: u = codes8<FP8_E5_A>(v, bq); break;
        }
        *(uint2*)(p.q8 + row * p.ldq8 + col) = u;
    }
    return mag8(v);
}

__device__ __forceinline__ uint4 scaled8(const float* a, float f) {
    return make_uint4(pack_bf16x2(a[0] * f, a[1] * f), pack_bf16x2(a[2] * f, a[3] * f), pack_bf16x2(a[4] * f, a[5] * f),
                      pack_bf16x2(a[6] * f, a[7] * f));
}
// Pairs of floats to and from where every XCD sees them.
__device__ __forceinline__ void put_far(uint64_t* p, float a, float b) {
    __hip_atomic_store(p, ((uint64_t)__float_as_uint(b) << 32) | __float_as_uint(a), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_far(uint64_t* p) {
    const uint64_t v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
// A partial (maximum and sum ml, output x, y) added to the sums relative to top.
__device__ __forceinline__ void add_part(float* acc, float& ll, float2 ml, float top, float c2, float4 x, float4 y) {
    if (ml.x == -INFINITY && ml.y == 0.0f) return;
    const float f = ml.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((ml.x - top) * c2);
    ll += f * ml.y;
    acc[0] += f * x.x;
    acc[1] += f * x.y;
    acc[2] += f * x.z;
    acc[3] += f * x.w;
    acc[4] += f * y.x;
    acc[5] += f * y.y;
    acc[6] += f * y.z;
    acc[7] += f * y.w;
}

// ---- up to 16 packed rows
// Wave w takes the steps w, w + kFewW, ... of its workgroup's keys: steps of 64 keys in
// FP8, 32 in bf16, 16 KB either way at d_head 128.  Of a step's four groups of G =
// 16 (8) keys, lane (r, g) = (lane % 16, lane / 16) reads for key tile kt the bytes
// 64 v + 16 g .. of key G (r / 4) + 4 kt + r % 4 (so that a load takes whole 64-byte
// pieces of rows; the queries have the same order of dimensions).  With this order
// of the rows, the scores that lane (q, g) gets are of the keys G g + 4 kt + i, whose
// values for dimension 16 dt + r it reads as one vector.  Nothing moves between
// lanes.  The cache is read once: its loads carry the non-temporal hint.  Bound by
// memory: 32 sequences of up to 16000 tokens, 64 heads on 8, in 95 us (5.2 TB/s; 16 to 64
// of 8000 to 16000 each 5.9 to 6.5, a plain sum over 1 GiB 6.0), 16 of up to 2500
// with 32 heads of their own in 32 us; one token over 300 in 7.5, mostly its loads in turn.
//
// Work: without `flat` a workgroup takes one item, a (sequence, key/value head), or
// where those are few one of few_parts equal parts of it.
// With it, the tiles of all items in a row are cut into equal shares, one for each
// workgroup: however ragged the lengths, every compute unit (whose loads run at
// some 35 GB/s at most) has the same work.  An item that several shares cut is joined by
// the one that finishes last.  The partials pass through device-scope atomic
// stores and loads, which the L2s of the XCDs do not hold back, and a count of the
// finished parts of the item, which is zero again when the call ends.
struct FewWork {
    int s, hk, nt;   // item, its tiles
    int64_t at;      // its first tile among all
    int per;         // tiles of a share
};
// Tiles of sequence s (0 if it is not few_body's, or sees no key).
__device__ __forceinline__ int few_tiles(const AttnArgs& p, int s) {
    const Seq sq = seq_of(p.c, s);
    const int m1 = min(sq.n, p.max_rows) * p.grp;
    return m1 < 1 || m1 > kFew ? 0 : range_of(p, sq, 0, m1, 0, 1).nt;
}
// The sequence of the k-th largest number of tiles, if there are up to 64;
// sequence k otherwise.  Workgroups take the longest items first, and those of the
// second one on a compute unit the shortest first, so that a long one has a short
// one beside it.
__device__ __forceinline__ int few_ranked(const AttnArgs& p, int k) {
    const int lane = threadIdx.x & 63, ns = p.c.n_seqs;
    if (ns > 64 || ns == 1) return k;
    const int mine = lane < ns ? few_tiles(p, lane) : -1;
    int rank = 0;
    for (int j = 0; j < ns; ++j) {
        const int x = __builtin_amdgcn_readlane(mine, j);
        rank += x > mine || (x == mine && j < lane);
    }
    return __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(lane < ns && rank == k)) - 1);
}
// Tiles of a share, and the item that the first tile of one falls into (nt 0: none).
__device__ __forceinline__ FewWork few_locate(const AttnArgs& p, int share, int shares) {
    const int lane = threadIdx.x & 63, ns = p.c.n_seqs, nkv = p.c.nkv;
    FewWork f = {0, 0, 0, 0, 0};
    int64_t total = 0;
    int mine = 0;  // tiles of this lane's sequence of the last 64 looked at
    int upto = 0;  // and of those before it, itself included (below 2^31: 64 times 2^24)
    auto look = [&](int s0) {
        upto = mine = s0 + lane < ns ? few_tiles(p, s0 + lane) : 0;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(upto, off, 64);
            upto += lane >= off ? y : 0;
        }
    };
    for (int s0 = 0; s0 < ns; s0 += 64) {
        look(s0);
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    total *= nkv;
    const int64_t per = (total + shares - 1) / shares;
    f.per = (int)(per < kShareLeast ? kShareLeast : per);
    const int64_t from = (int64_t)share * f.per;
    int64_t before = 0;
    for (int s0 = 0; s0 < ns && from < total; s0 += 64) {
        if (ns > 64) look(s0);
        const uint64_t beyond = __ballot((before + upto) * nkv > from);
        if (beyond) {
            const int k = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)beyond) - 1);
            f.s = s0 + k;
            f.nt = __builtin_amdgcn_readlane(mine, k);
            const int64_t start = (before + __builtin_amdgcn_readlane(upto, k) - f.nt) * nkv;
            f.hk = (int)((from - start) / f.nt);
            f.at = start + (int64_t)f.hk * f.nt;
            break;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return f;
}

template <int DH>
struct FewLds {
    float so[kFewW][kFew][DH + 4];
    float sm[kFewW][kFew], sl[kFewW][kFew];
    int last;
};
// Workgroup `wg` of `wgs`; returns the largest magnitude of what this thread wrote.
template <int FMT, int DH>
__device__ __forceinline__ uint32_t few_body(const AttnArgs& p, FewLds<DH>& lds, int wg, int wgs, bool cast, int bq) {
    constexpr int kE = FMT == kBf16 ? 1 : FMT;
    constexpr int kSteps = DH / 32;                    // of the contraction over d_head
    constexpr int kKv = DH * kEsz<FMT> / 64;           // 16-byte vectors of a lane's keys
    constexpr int kDt = DH / 16;                       // tiles of dimensions, a vector of values each
    constexpr int kG = 16 / kEsz<FMT>, kKeys = 4 * kG; // keys of a lane group, of a step
    constexpr int kKt = kG / 4, kPv = kG / 8;          // key tiles, steps of P . V
    constexpr int kCh = DH / 8;
    constexpr int kJoin = 8;                           // parts that are read at once
    static_assert(kFew * kCh <= kFewT, "a thread for eight values of a row");
    auto &so = lds.so;
    auto &sm = lds.sm, &sl = lds.sl;
    int& last = lds.last;
    const CacheView& c = p.c;
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
    // uniform to the compiler too: branches around matrix instructions, which
    // do not heed the lane mask, are then scalar
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rb = r16 >> 2, rl = r16 & 3;  // group and place of this lane's keys
    uint32_t mag = 0;
    FewWork f;
    const int items = c.n_seqs * c.nkv;
    int part = 0;
    int64_t at = 0, end = INT64_MAX;
    int kpage = -1, vpage = -1;  // of the next step to load
    bool any = true;
    if (p.flat) {
        f = few_locate(p, wg, wgs);
        at = (int64_t)wg * f.per;
        end = at + f.per;
        any = f.nt > 0;
    } else {
        int i = wg;
        if (p.few_parts > 1) {  // all run at once: in order
            part = i / items;
            i %= items;
            f.s = i / c.nkv;
        } else {
            if (items > kCus && items <= 2 * kCus && i >= kCus) i = items - 1 - (i - kCus);
            f.s = few_ranked(p, i / c.nkv);
        }
        f.hk = i % c.nkv;
        f.at = 0;
        f.per = INT32_MAX;
        // pages of the first step, before the lengths are there (used if the
        // keys turn out to start at 0)
        if (part == 0 && c.max_pages > 0) {
            const int32_t* row = c.pages + (int64_t)f.s * c.ld_pages;
            kpage = row[min((kKeys * w + kG * rb) >> c.page_shift, c.max_pages - 1)];
            vpage = row[min((kKeys * w + kG * g) >> c.page_shift, c.max_pages - 1)];
        }
    }
    while (any) {
        const int s = f.s, hk = f.hk;
        const Seq sq = seq_of(c, s);
        const int m1 = min(sq.n, p.max_rows) * p.grp;
        if (m1 < 1 || m1 > kFew) break;
        const Range rg = range_of(p, sq, 0, m1, 0, 1);
        int tb, te, live = 1;  // this workgroup's tiles, parts of the item without `flat`
        if (p.flat) {
            tb = (int)(at - f.at);
            te = (int)(end - f.at < rg.nt ? end - f.at : rg.nt);
        } else {
            live = max(min(p.few_parts, rg.nt / kFewPart), 1);
            const int each = (rg.nt + live - 1) / live;
            live = each > 0 ? (rg.nt + each - 1) / each : 1;
            tb = min(part * each, rg.nt);
            te = min(tb + each, rg.nt);
            if (part >= live && part > 0) break;
        }
        // this lane's query (rows past the last one repeat it, and are not stored)
        const int mq = min(r16, m1 - 1), tok = mq / p.grp;
        const int pos = sq.p0 + tok;
        const uint16_t* qp = p.q + (sq.r0 + tok) * p.ldq + (int64_t)(hk * p.grp + mq % p.grp) * DH;
        const int lo = p.window > 0 ? pos - p.window : -1;  // the last key before those that the row sees

        u32x4 kreg[kKt][kKv], vreg[kDt];
        u32x4 kex, vex;
        int64_t kbase, vbase;  // slots of the first keys of the two groups
        int vn;                // valid keys of the values' one (0 if the page is absent)
        auto page_in = [&](int t, int grp) {
            const int key = rg.start + kKeys * t + kG * grp;
            const int i = min(key >> c.page_shift, c.max_pages - 1);  // in the table, where the key is not
            return c.pages[(int64_t)s * c.ld_pages + i];
        };
        auto here = [&](int page) { return page >= 0 && page < c.n_pages; };
        auto where = [&](int t, int grp, int page) {
            return slot_of(c, here(page) ? page : 0, hk, rg.start + kKeys * t + kG * grp);
        };
        auto values_at = [&](int t, int page) {
            vbase = where(t, g, page);
            vn = here(page) ? max(min(rg.kend - (rg.start + kKeys * t + kG * g), kG), 0) : 0;
        };
        auto load_k = [&](int t) {
            kbase = where(t, rb, kpage);
            if (FMT != kBf16) kex = *(const u32x4*)(c.ke + kbase);
#pragma unroll
            for (int kt = 0; kt < kKt; ++kt)
#pragma unroll
                for (int v = 0; v < kKv; ++v)
                    kreg[kt][v] = __builtin_nontemporal_load(
                        (const u32x4*)(c.k + (kbase + 4 * kt + rl) * (DH * kEsz<FMT>) + 64 * v + 16 * g));
            kpage = page_in(t + kFewW, rb);
        };
        auto v_at = [&](int dt) {
            return c.v + ((vbase & ~(int64_t)(kBlk - 1)) * DH + (16 * dt + r16) * kBlk + (vbase & (kBlk - kG))) * kEsz<FMT>;
        };
        auto load_v = [&](int t) {
            values_at(t, vpage);
            if (FMT != kBf16) vex = *(const u32x4*)(c.ve + vbase);
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) vreg[dt] = __builtin_nontemporal_load((const u32x4*)v_at(dt));
            vpage = page_in(t + kFewW, g);
        };

        f4_t o[kDt];
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) o[dt] = f4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.0f;
        u32x4 qf[kSteps];
#pragma unroll
        for (int st = 0; st < kSteps; ++st)
            qf[st] = ldg16(qp + (FMT == kBf16 ? 32 * st + 8 * g : 64 * (st >> 1) + 16 * g + 8 * (st & 1)));
        // scores of the loaded tile (raw), and the masks of a tile at an edge
        auto scores = [&](f4_t (&sc)[kKt]) {
#pragma unroll
            for (int kt = 0; kt < kKt; ++kt) {
                sc[kt] = f4_t{0.f, 0.f, 0.f, 0.f};
                const float ks = FMT == kBf16 ? 1.0f : exp_float((kex[kt] >> (8 * rl)) & 0xFFu);
#pragma unroll
                for (int st = 0; st < kSteps; ++st) {
                    u32x4 kf;
                    if (FMT == kBf16) kf = kreg[kt][st];
                    else kf = cvt8b<kE>(kreg[kt][st / 2][2 * (st & 1)], kreg[kt][st / 2][2 * (st & 1) + 1], ks);
                    sc[kt] = mfma_bf16(kf, qf[st], sc[kt]);
                }
            }
        };
        auto is_edge = [&](int kb) {
            return kb + kKeys - 1 > rg.first || (p.window > 0 && kb <= rg.last - p.window) || __any(vn < kG);
        };
        // bit i: key i of this lane's group is seen by its row; keys lo + 1 .. lo +
        // seen are, if the page is present
        auto seen_bits = [&](int kb) {
            const int seen = vn > 0 ? max(min(pos, rg.kend - 1) - lo, 0) : 0, from = kb + kG * g - lo - 1;
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < kG; ++i) bits |= (unsigned)(from + i) < (unsigned)seen ? 1u << i : 0u;
            return bits;
        };
        // a 1 in the top bit of each value that is not finite
        auto nf = [](uint32_t x) {
            return FMT == kBf16 ? nonfinite2(x) : ((x & 0x7F7F7F7Fu) + (kE == FP8_E5M2 ? 0x04040404u : 0x01010101u)) & 0x80808080u;
        };
        auto vfrag = [&](u32x4 v, int st) {  // keys 8 st .. 8 st + 7 of this lane's group
            if (FMT == kBf16) return v;
            return cvt8b<kE>(v[2 * st & 3], v[(2 * st + 1) & 3], 1.0f);
        };

        bool hidden = false;  // infinities or NaN among the values of an edge
        const int tend = te * (kTile / kKeys), tfirst = tb * (kTile / kKeys) + w;
        int t = tfirst;
        if (t < tend) {
            if (tb > 0 || p.flat || p.window > 0) {
                kpage = page_in(t, rb);
                vpage = page_in(t, g);
            }
            load_k(t);
            load_v(t);
        }
        auto tile = [&](int kb, auto edge) {
            const bool more = t + kFewW < tend;  // its loads follow the last use of this tile's registers
            f4_t sc[kKt];
            scores(sc);
            if (more) load_k(t + kFewW);
            if (edge) {
                const uint32_t bits = seen_bits(kb);
#pragma unroll
                for (int i = 0; i < kG; ++i) sc[i >> 2][i & 3] = (bits >> i) & 1u ? sc[i >> 2][i & 3] : -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < kKt; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[kt][i]);
            mx = quad_max(mx);
            if (__any(mx > m)) {
                const float mn = fmaxf(m, mx);
                const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - mn) * p.c2);
                m = mn;
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < kDt; ++dt) o[dt] *= alpha;
            }
            const float moff = m == -INFINITY ? 0.0f : m;
            u32x4 pf[kPv];
#pragma unroll
            for (int kt = 0; kt < kKt; ++kt) {
                float pr[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // the difference first: its product with c2 is never above 0, however large the scores
                    pr[i] = __builtin_amdgcn_exp2f((sc[kt][i] - moff) * p.c2);
                    l += pr[i];
                    if (FMT != kBf16) pr[i] *= exp_float((vex[kt] >> (8 * i)) & 0xFFu);
                }
                pf[kt >> 1][2 * (kt & 1)] = pack_bf16x2(pr[0], pr[1]);
                pf[kt >> 1][2 * (kt & 1) + 1] = pack_bf16x2(pr[2], pr[3]);
            }
            if (!edge) {
#pragma unroll
                for (int st = 0; st < kPv; ++st)
#pragma unroll
                    for (int dt = 0; dt < kDt; ++dt) o[dt] = mfma_bf16(vfrag(vreg[dt], st), pf[st], o[dt]);
            } else {
                uint32_t mk[4], any = 0;
                token_masks<kG / 4>(vn, mk);  // slots that hold no token may hold NaN
#pragma unroll
                for (int dt = 0; dt < kDt; ++dt) {
                    u32x4 v = vreg[dt];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t x = v[k] & mk[k], bad = nf(x);
                        any |= bad;
                        v[k] = x & ~((bad >> (FMT == kBf16 ? 15 : 7)) * (FMT == kBf16 ? 0xFFFFu : 0xFFu));
                    }
                    // the finite part here, what the rest adds below
#pragma unroll
                    for (int st = 0; st < kPv; ++st) o[dt] = mfma_bf16(vfrag(v, st), pf[st], o[dt]);
                }
                hidden = hidden || __any(any);
            }
            if (more) load_v(t + kFewW);
        };
        for (; t < tend; t += kFewW) {
            const int kb = rg.start + kKeys * t;
            tile(kb, is_edge(kb));
        }
        if (hidden) {
#pragma unroll 1
            for (t = tfirst; t < tend; t += kFewW) {
                const int kb = rg.start + kKeys * t;
                values_at(t, page_in(t, g));
                if (!is_edge(kb)) continue;
                const uint32_t bits = seen_bits(kb);
                uint32_t mk[4];
                token_masks<kG / 4>(vn, mk);
#pragma unroll
                for (int dt = 0; dt < kDt; ++dt) {  // one operand at a time: few registers
                    u32x4 vv = *(const u32x4*)v_at(dt);
#pragma unroll
                    for (int k = 0; k < 4; ++k) vv[k] &= mk[k];
#pragma unroll
                    for (int st = 0; st < kPv; ++st) {
                        u32x4 up, down;
                        split_nonfinite(vfrag(vv, st), up, down);
                        const u32x4 wm = ones_where(bits >> (8 * st));
                        const f4_t zero = {0.f, 0.f, 0.f, 0.f};
                        const f4_t cu = mfma_bf16(up, wm, zero), cd = mfma_bf16(down, wm, zero);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[dt][i] = add_nonfinite(o[dt][i], cu[i], cd[i]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        l = quad_sum(l);
        // join the waves
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) *(f4_t*)&so[w][r16][16 * dt + 4 * g] = o[dt];
        if (g == 0) {
            sm[w][r16] = m;
            sl[w][r16] = l;
        }
        __syncthreads();
        const int row = tid / kCh, ch = tid % kCh;
        const bool mine = row < m1;
        float mm = -INFINITY, acc[8], ll = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        if (mine) {
#pragma unroll
            for (int k = 0; k < kFewW; ++k) mm = fmaxf(mm, sm[k][row]);
#pragma unroll
            for (int k = 0; k < kFewW; ++k) {
                const float* x = &so[k][row][8 * ch];
                add_part(acc, ll, make_float2(sm[k][row], sl[k][row]), mm, p.c2, *(const float4*)x, *(const float4*)(x + 4));
            }
        }
        bool write = true;
        if (tb > 0 || te < rg.nt) {
            // d_head outputs and (maximum, sum) of kFew rows: without `flat` [part][item]; with it
            // [share][2], the part of an item that starts in the share in 1, of one
            // that started before in 0
            const int64_t w0 = p.flat ? f.at / f.per : 0, w1 = p.flat ? (f.at + rg.nt - 1) / f.per : live - 1;
            uint64_t* po = (uint64_t*)p.few_o + row * (DH / 2) + 4 * ch;
            uint64_t* pm = (uint64_t*)p.few_ml + row;
            auto slot = [&](int64_t k) {
                return (p.flat ? 2 * k + (k == w0) : k * items + s * c.nkv + hk) * kFew;
            };
            const int64_t own = slot(p.flat ? wg : part);
            if (mine) {
#pragma unroll
                for (int e = 0; e < 4; ++e) put_far(po + own * (DH / 2) + e, acc[2 * e], acc[2 * e + 1]);
                if (ch == 0) put_far(pm + own, mm, ll);
            }
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");  // they are where every XCD sees them
            __syncthreads();
            if (tid == 0) {
                int32_t* count = p.counts + (int64_t)s * c.nkv + hk;
                const int done = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last = done == w1 - w0;
                if (last) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            write = last;
            if (write && mine) {
                mm = -INFINITY;
                ll = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
                // several parts' loads at once: each takes a trip to memory.  (Those
                // behind the last part read it again, with no weight.)
                for (int64_t k0 = w0; k0 <= w1; k0 += kJoin) {
                    float2 ml[kJoin], x[kJoin][4];
#pragma unroll
                    for (int k = 0; k < kJoin; ++k) {
                        const int64_t sl = slot(min(k0 + k, w1));
                        ml[k] = get_far(pm + sl);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[k][e] = get_far(po + sl * (DH / 2) + e);
                    }
                    float top = mm;
#pragma unroll
                    for (int k = 0; k < kJoin; ++k) {
                        if (k0 + k > w1) ml[k] = make_float2(-INFINITY, 0.0f);
                        top = fmaxf(top, ml[k].x);
                    }
                    const float f = mm == -INFINITY ? (top == -INFINITY ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f((mm - top) * p.c2);
                    mm = top;
                    if (ll != 0.0f) {
                        ll *= f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[e] *= f;
                    }
#pragma unroll
                    for (int k = 0; k < kJoin; ++k)
                        add_part(acc, ll, ml[k], mm, p.c2, make_float4(x[k][0].x, x[k][0].y, x[k][1].x, x[k][1].y),
                                 make_float4(x[k][2].x, x[k][2].y, x[k][3].x, x[k][3].y));
                }
            }
        }
        if (write && mine)
            mag = max(mag, put8(p, cast, bq, sq.r0 + row / p.grp, (int64_t)(hk * p.grp + row % p.grp) * DH + 8 * ch,
                                scaled8(acc, ll == 0.0f ? 0.0f : 1.0f / ll)));
        if (!p.flat) break;
        at = f.at += rg.nt;
        if (++f.hk == c.nkv) {  // the next sequence that has tiles
            f.hk = 0;
            f.nt = 0;
            while (f.nt == 0 && ++f.s < c.n_seqs) f.nt = few_tiles(p, f.s);
        }
        any = f.nt > 0 && at < end;
        __syncthreads();  // the next item writes to the shared memory
    }
    // items that see no key have no tiles: one share writes their zeros
    if (p.flat)
        for (int s = wg; s < c.n_seqs; s += wgs) {
            const Seq sq = seq_of(c, s);
            const int n = min(sq.n, p.max_rows), cols = p.nh * DH / 8;
            if (n < 1 || n * p.grp > kFew || few_tiles(p, s) > 0) continue;
            for (int i = tid; i < n * cols; i += kFewT)
                put8(p, cast, bq, sq.r0 + i / cols, 8 * (i % cols), make_uint4(0u, 0u, 0u, 0u));
        }
    return mag;
}

// ---- tiles of 128 packed rows
// Wave w owns packed rows 32 w .. 32 w + 31 of the tile, one per lane pair (the
// queries stay in registers).  Tiles of 64 keys are double-buffered in LDS as
// bf16: wave w brings in the 16 keys of block w, converts the codes on the way
// (once for the four waves) and loads the tile after next meanwhile.
//   K: rows of one key, 16-byte chunk c at c ^ (key mod 16 or 8);
//   V: rows of one dimension, 64 keys each, a block's keys in the order 0-3,
//      8-11, 4-7, 12-15 that the scores' registers have; chunk c at
//      c ^ (d / 2 mod 8).  Any 16 rows of one chunk then cover the 64 banks.
// Score register i of lane (q, h) is key 8 (i / 4) + 4 h + i % 4 of 32.
//
// Bound by what two waves a SIMD overlap of 32 matrix instructions (a third of the
// time), 291 vector instructions (as long) and 51 of LDS (as long) a tile, at d_head
// 128 in E4M3: 512 tokens over 8192 before them, 64 heads on 8, in 176 to 182 us
// (805 to 780 TFLOP/s; a library product of 8192^3 runs at 1190), 2 x 2048 tokens of 32
// heads in bf16 in 104 to 109 (660 to 630; the attention within a call, which has whole
// sequences and no pages, takes 81).  Measured and left: software pipelining within a wave (spills at
// 128; 122 us against 128 at 64), matrix instructions on FP8 operands (see above).
template <int DH>
struct ManyLds {
    uint8_t __attribute__((aligned(16))) kv[4 * kTile * DH * 2];  // K0 V0 K1 V1; output staging
    float __attribute__((aligned(16))) vsc[2][kTile];             // 2^(exp - 127) of the values
    int __attribute__((aligned(16))) info[2][4];                  // valid keys of a block
    int hidden;                                                   // sums came out nonfinite
};
// Workgroup `wg` of `wgs`; returns the largest magnitude of what this thread wrote.
template <int FMT, int DH>
__device__ __forceinline__ uint32_t many_body(const AttnArgs& p, ManyLds<DH>& shared, int wg, int wgs, bool cast, int bq) {
    constexpr int kE = FMT == kBf16 ? 1 : FMT;
    constexpr int kSteps = DH / 16;                       // of the contraction over d_head
    constexpr int kDt = DH / 32;                          // tiles of dimensions
    constexpr int kKb = kTile * DH * 2;                   // bytes of K (and of V) in LDS
    constexpr int kKmask = DH / 8 - 1;                    // chunks of a key row, less one
    constexpr int kKv = DH * kEsz<FMT> / 64;              // 16-byte vectors of keys a lane brings in
    constexpr int kVd = DH / 64;                          // dimensions whose values it brings in
    constexpr int kVv = kEsz<FMT>;                        // vectors of each
    enum { kAll, kFinite, kRest };                        // sweeps over the keys: of all values, or in two
    auto& lds = shared.kv;
    auto& vsc = shared.vsc;
    auto& info = shared.info;
    int& hidden = shared.hidden;
    const CacheView& c = p.c;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    const int hk = wg % c.nkv;
    int rest = wg / c.nkv;
    const int split = rest % p.splits;
    rest = wgs / (c.nkv * p.splits) - 1 - rest / p.splits;  // the last rows, with the longest ranges, first
    // tile slots: as many for each sequence as cu_rows[s + 1] / kMany + 1 - cu_rows[s] / kMany in packed rows
    const int s = wave_search(c.n_seqs, rest, [&](int i) { return row_at(c, i) * p.grp / kMany + i; });
    const Seq sq = seq_of(c, s);
    const int m0 = (int)(rest - (sq.r0 * p.grp / kMany + s)) * kMany;
    const int mtot = min(sq.n, p.max_rows) * p.grp;
    const int m1 = min(m0 + kMany, mtot);
    const Range rg = range_of(p, sq, min(m0, mtot), max(m1, 1), split, p.per);
    // (below 0 only where cu_rows does not start with 0)
    if (m0 < 0 || m0 >= mtot || (p.few_on && mtot <= kFew) || (split > 0 && rg.t0 >= rg.t1))
        return 0u;
    const int mq = min(m0 + 32 * w + l32, m1 - 1), tok = mq / p.grp;
    const int pos = sq.p0 + tok;
    const uint16_t* qp = p.q + (sq.r0 + tok) * p.ldq + (int64_t)(hk * p.grp + mq % p.grp) * DH;
    u32x4 qf[kSteps];
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) qf[ks] = ldg16(qp + 16 * ks + 8 * h);

    const int lo = p.window > 0 ? pos - p.window : -1;  // the last key before those that the row sees
    const int seen = max(min(pos, rg.kend - 1) - lo, 0);

    // this wave's block of a tile: raw codes on their way to LDS
    u32x4 kraw[kKv], vraw[kVd][kVv];
    uint32_t ke = 0, ve = 0;
    int nval = 0;
    auto page_at = [&](int t) {
        const int b0 = rg.start + kTile * t + kBlk * w;
        return b0 < rg.kend ? page_of(c, s, b0) : -1;
    };
    auto load = [&](int t, int page) {
        const int b0 = rg.start + kTile * t + kBlk * w;
        nval = page >= 0 ? min(rg.kend - b0, kBlk) : 0;
        const int64_t slot = slot_of(c, max(page, 0), hk, b0);
        const uint8_t* kp = c.k + (slot + (lane >> 2)) * (DH * kEsz<FMT>) + (lane & 3) * (DH / 4) * kEsz<FMT>;
#pragma unroll
        for (int v = 0; v < kKv; ++v) kraw[v] = *(const u32x4*)(kp + 16 * v);
#pragma unroll
        for (int d = 0; d < kVd; ++d)
#pragma unroll
            for (int v = 0; v < kVv; ++v)
                vraw[d][v] = *(const u32x4*)(c.v + (slot * DH + (lane + 64 * d) * kBlk) * kEsz<FMT> + 16 * v);
        if (FMT != kBf16) {
            ke = c.ke[slot + (lane >> 2)];
            ve = c.ve[slot + (lane & 15)];
        }
    };
    // mode kFinite: infinities and NaN among the values left out
    auto store = [&](int buf, auto mode) {
        uint8_t* Kl = lds + buf * 2 * kKb;
        uint8_t* Vl = Kl + kKb;
        const int key = kBlk * w + (lane >> 2);
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
            u32x4 x;
            if (FMT == kBf16) x = kraw[j % kKv];
            else x = cvt8b<kE>(kraw[j / 2 % kKv][2 * (j & 1)], kraw[j / 2 % kKv][2 * (j & 1) + 1], exp_float(ke));
            const int ch = (lane & 3) * (DH / 32) + j;
            *(u32x4*)(Kl + key * DH * 2 + ((ch ^ (key & kKmask)) << 4)) = x;
        }
        const int n = nval;
        if (n < kBlk) {  // slots that hold no token may hold NaN
            uint32_t mk[4 * kVv];
            token_masks<4 / kEsz<FMT>>(n, mk);
#pragma unroll
            for (int d = 0; d < kVd; ++d)
#pragma unroll
                for (int k = 0; k < 4 * kVv; ++k) vraw[d][k / 4][k % 4] &= mk[k];
        }
        if constexpr (mode == kFinite) {
            // a 1 in the top bit of each value that is not finite
            auto nf = [](uint32_t x) {
                return FMT == kBf16 ? nonfinite2(x) : ((x & 0x7F7F7F7Fu) + (kE == FP8_E5M2 ? 0x04040404u : 0x01010101u)) & 0x80808080u;
            };
#pragma unroll
            for (int d = 0; d < kVd; ++d)
#pragma unroll
                for (int k = 0; k < 4 * kVv; ++k) {
                    const uint32_t x = vraw[d][k / 4][k % 4];
                    vraw[d][k / 4][k % 4] = x & ~((nf(x) >> (FMT == kBf16 ? 15 : 7)) * (FMT == kBf16 ? 0xFFFFu : 0xFFu));
                }
        }
#pragma unroll
        for (int d = 0; d < kVd; ++d) {
            u32x4 x[2];
            const u32x4 v0 = vraw[d][0], v1 = vraw[d][kVv - 1];
            if (FMT == kBf16) {
                x[0] = u32x4{v0[0], v0[1], v1[0], v1[1]};
                x[1] = u32x4{v0[2], v0[3], v1[2], v1[3]};
            } else {
                x[0] = cvt8b<kE>(v0[0], v0[2], 1.0f);
                x[1] = cvt8b<kE>(v0[1], v0[3], 1.0f);
            }
            const int dim = lane + 64 * d;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *(u32x4*)(Vl + dim * (kTile * 2) + (((2 * w + e) ^ ((dim >> 1) & 7)) << 4)) = x[e];
        }
        if (FMT != kBf16 && lane < kBlk) vsc[buf][kBlk * w + lane] = lane < n ? exp_float(ve) : 0.0f;
        if (lane == 0) info[buf][w] = n;
    };

    f16_t o[kDt];
    float m, l;
    auto start = [&]() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
    };
    start();
    const float lazy = 8.0f / p.c2;
    bool apart = false;  // this row takes differences of scores first

    auto sweep = [&](auto mode) {
        int page = page_at(rg.t0);
        load(rg.t0, page);
        page = page_at(min(rg.t0 + 1, rg.t1 - 1));
        store(0, mode);
        load(min(rg.t0 + 1, rg.t1 - 1), page);
        page = page_at(min(rg.t0 + 2, rg.t1 - 1));
        __syncthreads();
        for (int t = rg.t0; t < rg.t1; ++t) {
            const int buf = (t - rg.t0) & 1;
            const uint8_t* Kl = lds + buf * 2 * kKb;
            const uint8_t* Vl = Kl + kKb;
            auto kfrag = [&](int ks, int kt) {
                const int key = 32 * kt + l32;
                return *(const u32x4*)(Kl + key * DH * 2 + (((2 * ks + h) ^ (key & kKmask)) << 4));
            };
            auto vfrag = [&](int dt, int b) {
                const int dim = 32 * dt + l32;
                return *(const u32x4*)(Vl + dim * (kTile * 2) + (((2 * b + h) ^ ((dim >> 1) & 7)) << 4));
            };
            // The first key operands are under way while the next tile goes into
            // the other buffer, which every wave has finished reading (after the
            // last tile it is written once more for nothing), the others while
            // the first products run.
            u32x4 kf[kSteps / 2][2];
#pragma unroll
            for (int ks = 0; ks < kSteps / 2; ++ks)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) kf[ks][kt] = kfrag(ks, kt);
            __builtin_amdgcn_sched_barrier(0);
            store(buf ^ 1, mode);
            load(min(t + 2, rg.t1 - 1), page);
            page = page_at(min(t + 3, rg.t1 - 1));
            f16_t sc[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[kt][i] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    sc[kt] = mfma32(kf[ks % (kSteps / 2)][kt], qf[ks], sc[kt]);
                    if (ks < kSteps / 2) kf[ks][kt] = kfrag(ks + kSteps / 2, kt);
                }
            const int4 in4 = *(const int4*)info[buf];
            const int in[4] = {__builtin_amdgcn_readfirstlane(in4.x), __builtin_amdgcn_readfirstlane(in4.y),
                               __builtin_amdgcn_readfirstlane(in4.z), __builtin_amdgcn_readfirstlane(in4.w)};
            const int kb = rg.start + kTile * t;
            const bool full = ((in[0] & in[1] & in[2] & in[3]) & kBlk) != 0;
            if (!full || kb + kTile - 1 > rg.first || (p.window > 0 && kb <= rg.last - p.window)) {
                // keys lo + 1 .. lo + seen are seen, of blocks whose page is present
                const int from = kb + 4 * h - lo - 1;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const unsigned n = in[b] ? seen : 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = 8 * (b & 1) + i;
                        const bool see = (unsigned)(from + 16 * b + 8 * (i >> 2) + (i & 3)) < n;
                        sc[b >> 1][at] = see ? sc[b >> 1][at] : -INFINITY;
                    }
                }
            }
            if constexpr (mode != kRest) {
                u32x4 vf[2][kDt];  // the first value operands, under way during the softmax
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int dt = 0; dt < kDt; ++dt) vf[b][dt] = vfrag(dt, b);
                __builtin_amdgcn_sched_barrier(0);
                float mx = -INFINITY;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[kt][i]);
                {
                    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                    mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
                }
                // the exponent offset moves only when a score exceeds it by 2^8 in
                // probability: rarely, and never by more than what fp32 and bf16 hold
                const bool grow = mx > m + lazy;
                if (__any(grow)) {
                    const float mn = grow ? mx : m;
                    const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - mn) * p.c2);
                    m = mn;
                    l *= alpha;
#pragma unroll
                    for (int dt = 0; dt < kDt; ++dt) o[dt] *= alpha;
                }
                const float mref = m == -INFINITY ? 0.0f : m, moff = -mref * p.c2;
                u32x4 pf[4];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        float pr[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float s = sc[kt][4 * q4 + i];
                            pr[i] = __builtin_amdgcn_exp2f(mode == kFinite && apart ? (s - mref) * p.c2 : fmaf(s, p.c2, moff));
                            l += pr[i];
                        }
                        if (FMT != kBf16) {
                            const f4_t vs = *(const f4_t*)&vsc[buf][32 * kt + 8 * q4 + 4 * h];
#pragma unroll
                            for (int i = 0; i < 4; ++i) pr[i] *= vs[i];
                        }
                        pf[2 * kt + (q4 >> 1)][2 * (q4 & 1)] = pack_bf16x2(pr[0], pr[1]);
                        pf[2 * kt + (q4 >> 1)][2 * (q4 & 1) + 1] = pack_bf16x2(pr[2], pr[3]);
                    }
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int dt = 0; dt < kDt; ++dt) {
                        o[dt] = mfma32(vf[b & 1][dt], pf[b], o[dt]);
                        if (b < 2) vf[b][dt] = vfrag(dt, b + 2);
                    }
            } else {
                // what infinities and NaN among the values add to the rows that see them
#pragma unroll 1
                for (int b = 0; b < 4; ++b) {
                    uint32_t bits = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) bits |= sc[0][i] == -INFINITY ? 0u : 1u << i;
                    const u32x4 wm = ones_where(bits);
#pragma unroll
                    for (int dt = 0; dt < kDt; ++dt) {
                        u32x4 up, down;
                        split_nonfinite(vfrag(dt, b), up, down);
#pragma unroll
                        for (int sgn = 0; sgn < 2; ++sgn) {
                            f16_t cnt;
#pragma unroll
                            for (int i = 0; i < 16; ++i) cnt[i] = 0.0f;
                            cnt = mfma32(sgn ? down : up, wm, cnt);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[dt][i] += cnt[i] > 0.0f ? (sgn ? -INFINITY : INFINITY) : 0.0f;
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sc[0][i] = sc[0][8 + i];
                        sc[0][8 + i] = sc[1][i];
                        sc[1][i] = sc[1][8 + i];
                    }
                }
            }
            __syncthreads();
        }
    };
    if (rg.t0 < rg.t1) {
        if (tid == 0) hidden = 0;
        // An infinity or NaN among the values makes sums of every row nonfinite, of
        // those that do not see it too (0 * NaN).  The loop does not look for them
        // (which cost 2 % of the call); where a sum comes out nonfinite, others do
        // it again: two with the finite values, one that adds what the rest gives
        // to the rows that see it.  Large scores need them too: the product of the
        // maximum with c2 is rounded, by up to 2^-24 of itself, and the row's weights
        // before and after a new maximum are off by as many powers of two: to zeros,
        // to infinities, or in between.  Rows whose product ends above 2^14 take the
        // difference first.  (Below, the rounding is 2^-11, a fraction of that of the
        // probabilities.  A maximum that was above 2^15 on the way and is not at the end
        // left weights of 0, infinities or NaN behind; rows where the latter stay
        // nonfinite take the difference in the second sweep.)  Four sweeps in place of one.
        auto nonfinite = [&]() {  // any of this lane's sums
            bool bad = !(l < INFINITY);
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) bad |= !(fabsf(o[dt][i]) < INFINITY);
            return bad;
        };
        sweep(IC<kAll>{});
        apart = m != -INFINITY && fabsf(m) * p.c2 > kLargeScore;
        if (__any(nonfinite() || apart)) hidden = 1;
        __syncthreads();
        if (hidden) {
            for (int again = 0; again < 2; ++again) {
                start();
                sweep(IC<kFinite>{});
                const int bad = nonfinite();
                apart = apart || bad || __shfl_xor(bad, 32, 64);  // the lanes of a row alike
            }
            sweep(IC<kRest>{});
        }
    }
    {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    if (p.splits > 1) {
        if (m0 + 32 * w + l32 < m1) {
            const int64_t at = ((int64_t)split * c.rows + sq.r0 + tok) * p.nh + hk * p.grp + mq % p.grp;
            if (h == 0) p.many_ml[at] = make_float2(m, l);
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
                    *(float4*)(p.many_o + at * DH + 32 * dt + 8 * q4 + 4 * h) =
                        make_float4(o[dt][4 * q4], o[dt][4 * q4 + 1], o[dt][4 * q4 + 2], o[dt][4 * q4 + 3]);
        }
        return 0u;
    }
    // rows of this head's d_head values through LDS (16-byte chunk c of row r at c ^ r)
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int rl = 32 * w + l32;
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int ch = 4 * dt + q4;
            *(uint2*)(lds + rl * DH * 2 + ((ch ^ (rl & kKmask)) << 4) + 8 * h) =
                make_uint2(pack_bf16x2(o[dt][4 * q4] * inv, o[dt][4 * q4 + 1] * inv),
                           pack_bf16x2(o[dt][4 * q4 + 2] * inv, o[dt][4 * q4 + 3] * inv));
        }
    __syncthreads();
    uint32_t mag = 0;
    constexpr int kCh = DH / 8;
    for (int i = tid; i < (m1 - m0) * kCh; i += kT) {
        const int row = i / kCh, ch = i % kCh, mm = m0 + row;
        const uint4 v = *(const uint4*)(lds + row * DH * 2 + ((ch ^ (row & kKmask)) << 4));
        mag = max(mag, put8(p, cast, bq, sq.r0 + mm / p.grp, (int64_t)(hk * p.grp + mm % p.grp) * DH + 8 * ch, v));
    }
    return mag;
}

// The counts of a call with the fused quantise, whose workspace other fused calls may have
// written (a launch of 1.6 us, only where items are cut: a count that does not start
// from zero never says which part is the last, and the item's rows stay unwritten).
__global__ __launch_bounds__(kT) void clear_kernel(int32_t* counts, int n) {
    const int i = blockIdx.x * kT + threadIdx.x;
    if (i < n) counts[i] = 0;
}

// The kernels.  Both in one launch where a call may have sequences of either kind:
// the latency of the one is then under the work of the other.
// Waves a SIMD: three where many_body's registers suffice (40 sequences of 128 rows
// over 960 keys, 12 heads of 64, E4M3: 44 us, with two 60).  With few_body beside it three
// are slower where single tokens have most of the keys (24 sequences over 2500,
// five of 200 rows, bf16: 66 us against 54), faster where few have (35 against 39).
template <int DH, bool MANY, bool FEW>
constexpr int kWaves = DH == 64 && MANY && !FEW ? 3 : 2;
template <int FMT, int DH, bool MANY, bool FEW>
__global__ __launch_bounds__(kT, (kWaves<DH, MANY, FEW>)) void attn_kernel(AttnArgs p) {
    static_assert(kFewT == kT, "one launch for both");
    __shared__ union Lds {
        __device__ Lds() {}
        ManyLds<MANY ? DH : 0> many;
        FewLds<FEW ? DH : 0> few;
    } lds;
    __shared__ uint32_t redm[kT / 64];
    const bool cast = p.q8 && p.pred;
    const int bq = p.q8 ? fused_bias(p.pred, p.used) : 0;
    const int wg = blockIdx.x;
    uint32_t mag = 0;
    if constexpr (MANY) {
        if (!FEW || wg < p.many_wg) mag = many_body<FMT, DH>(p, lds.many, wg, p.many_wg, cast, bq);
    }
    if constexpr (FEW) {
        const int before = MANY ? p.many_wg : 0;
        if (wg >= before) mag = few_body<FMT, DH>(p, lds.few, wg - before, gridDim.x - before, cast, bq);
    }
    if (p.q8) {
        const uint32_t bm = block_max(mag, redm);
        if (threadIdx.x == 0) p.parts[wg] = bm;
    }
}

// ---- join of the key ranges of many_body's rows, one (row, head) by DH / 8 lanes
template <int DH>
__global__ __launch_bounds__(kT) void many_join_kernel(AttnArgs p) {
    constexpr int kCh = DH / 8;
    __shared__ uint32_t redm[kT / 64];
    const CacheView& c = p.c;
    const bool cast = p.q8 && p.pred;
    const int bq = p.q8 ? fused_bias(p.pred, p.used) : 0;
    const uint32_t first = blockIdx.x * (kT / kCh), item = first + threadIdx.x / kCh;  // below 2^29: 2^24 workgroups
    const int ch = threadIdx.x % kCh;
    const int64_t r = item / (uint32_t)p.nh;
    const int head = (int)(item % (uint32_t)p.nh);
    uint32_t mag = 0;
    // The first two partials of the row are under way while its sequence is looked
    // for (there are two at least; in rows of few_body they are not used): 1700 rows
    // of 12 heads of 64, two partials, 6.2 -> 5.3 us.
    const int64_t step = c.rows * p.nh, at = min(r, c.rows - 1) * p.nh + head;
    float2 ml[2];
    float4 x[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float* d = p.many_o + (k * step + at) * DH + 8 * ch;
        ml[k] = p.many_ml[k * step + at];
        x[k][0] = *(const float4*)d;
        x[k][1] = *(const float4*)(d + 4);
    }
    // a workgroup's rows can lie in two sequences or more
    int s = wave_search(c.n_seqs, first / (uint32_t)p.nh, [&](int i) { return row_at(c, i); });
    while (s + 1 < c.n_seqs && row_at(c, s + 1) <= r) ++s;
    const Seq sq = seq_of(c, s);
    const int i = (int)(r - sq.r0), mtot = min(sq.n, p.max_rows) * p.grp;
    if (r < c.rows && i >= 0 && i * p.grp < mtot && !(p.few_on && mtot <= kFew)) {
        const int m0 = (i * p.grp + head % p.grp) / kMany * kMany;
        const Range rg = range_of(p, sq, m0, min(m0 + kMany, mtot), 0, p.per);
        float top = -INFINITY, acc[8], ll = 0.0f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k >= rg.live) ml[k] = make_float2(-INFINITY, 0.0f);
            top = fmaxf(top, ml[k].x);
        }
        for (int k = 2; k < rg.live; ++k) top = fmaxf(top, p.many_ml[k * step + at].x);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < 2; ++k) add_part(acc, ll, ml[k], top, p.c2, x[k][0], x[k][1]);
#pragma unroll 2
        for (int k = 2; k < rg.live; ++k) {
            const float* d = p.many_o + (k * step + at) * DH + 8 * ch;
            add_part(acc, ll, p.many_ml[k * step + at], top, p.c2, *(const float4*)d, *(const float4*)(d + 4));
        }
        mag = put8(p, cast, bq, r, (int64_t)head * DH + 8 * ch, scaled8(acc, ll == 0.0f ? 0.0f : 1.0f / ll));
    }
    if (p.q8) {
        const uint32_t bm = block_max(mag, redm);
        if (threadIdx.x == 0) p.parts[blockIdx.x] = bm;
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

// Heads of a group, so that about kBlockWgs workgroups run: a multiple of `per`, the
// heads that a workgroup takes of a whole block at a time.
static int group_heads(int64_t slots, int heads, int per) {
    const int64_t groups = slots < kBlockWgs ? kBlockWgs / slots : 1;
    const int64_t h = (heads + groups - 1) / groups;
    return (int)((h + per - 1) / per * per);
}

int32_t launch_cache_append(const uint16_t* qkv, int64_t ld, int nh, const CacheView& c, int fmt, int d_head,
                            const float* table, uint16_t* q, int64_t ldq, hipStream_t s) {
    const int per = kT / d_head, qk = (q ? nh : 0) + c.nkv;
    const int64_t slots = block_slots(c.rows, c.n_seqs);
    const int hqk = group_heads(slots, qk + c.nkv, per), hv = hqk < c.nkv ? hqk : (c.nkv + per - 1) / per * per;
    const int gqk = (qk + hqk - 1) / hqk, gv = (c.nkv + hv - 1) / hv;
    const dim3 grid((unsigned)slots, (unsigned)(gqk + gv));
    with_cache(fmt, d_head, [&](auto F, auto D) {
        hipLaunchKernelGGL((append_kernel<decltype(F)::value, decltype(D)::value>), grid, dim3(kT), 0, s, c, qkv, ld, nh,
                           (const float2*)table, q, ldq, gqk, hqk, hv);
    });
    return hip_status();
}

int32_t launch_cache_read(const CacheView& c, int fmt, int d_head, uint16_t* k, int64_t ldk, uint16_t* v, int64_t ldv,
                          hipStream_t s) {
    const int64_t slots = block_slots(c.rows, c.n_seqs);
    const int h = group_heads(slots, 2 * c.nkv, kT / d_head), g = (c.nkv + h - 1) / h;
    const dim3 grid((unsigned)slots, (unsigned)((k ? g : 0) + (v ? g : 0)));
    with_cache(fmt, d_head, [&](auto F, auto D) {
        hipLaunchKernelGGL((read_kernel<decltype(F)::value, decltype(D)::value>), grid, dim3(kT), 0, s, c, k, ldk, v, ldv,
                           k ? g : 0, h);
    });
    return hip_status();
}

namespace {
// How a call is split over workgroups, from its sizes alone.
struct Plan {
    bool few, many, flat;  // which kernels run, and few_body in shares
    int few_parts;         // or in parts of an item
    int splits, per;       // many_body's key ranges, and tiles of each
    int64_t few_wg, many_wg, many_join;
    int64_t parts, room;   // workgroups that write outputs; at most, whatever the window
    // offsets in the workspace, in bytes, behind the counts: words of the quantise, partials of either kernel
    int64_t words, few_o, few_ml, many_o, many_ml, ws_bytes;
};
Plan plan_of(int64_t rows, int nh, int nkv, int d_head, int64_t n_seqs, int64_t max_rows, int64_t max_len, int64_t window) {
    Plan p;
    const int64_t grp = nh / nkv, cap = max_rows < rows ? max_rows : rows;
    const int64_t tiles = (max_len + kTile - 1) / kTile;
    p.many = cap * grp > kFew;
    // sequences of one length have no single tokens among them
    p.few = !p.many || (grp <= kFew && n_seqs > 1 && rows < n_seqs * cap);
    const int64_t items = n_seqs * nkv;
    // few_body.  Shares where a compute unit would have much to read and the
    // items are few enough to be uneven (measured: 32 sequences of up to 16000
    // tokens, 8 heads, 97 us against 126 with an item a workgroup; but 16 of up to 2500, 32 heads, 81
    // against 32).  Lengths are on the device: the rule goes by the table's, and those 16
    // take shares too where it holds 4096 positions.  Parts where items would leave compute units idle: about
    // sqrt(2 tiles) of them, since a part costs the join what half a tile costs
    // its reader (one of 30000 tokens, 8 heads: 469 tiles, 29 parts 26 us, 64 parts 36).
    p.flat = p.few && items <= kCounts && n_seqs <= kFlatSeqs && items < 8 * kCus && tiles >= kFlatTiles &&
             items * tiles >= kShares * kFlatTiles;
    p.few_parts = 1;
    if (!p.flat && items < kCus) {
        const int64_t room = 2 * kCus / items, most = tiles / kFewPart;
        p.few_parts = (int)(room < most ? room : most);
        while ((int64_t)p.few_parts * p.few_parts > 2 * tiles) --p.few_parts;
        if (p.few_parts < 1) p.few_parts = 1;
    }
    p.few_wg = !p.few ? 0 : p.flat ? kShares : items * p.few_parts;
    // many_body: as many ranges as give kManyWant workgroups if all sequences
    // were of the longest length, of at least kManyLeast tiles
    const int64_t wg = (rows * grp / kMany + n_seqs) * nkv;
    int64_t seen = tiles;  // of a tile of rows
    if (window > 0 && (window + kMany / grp) / kTile + 2 < tiles) seen = (window + kMany / grp) / kTile + 2;
    int64_t most = (kManyWant + wg - 1) / wg, least = tiles / kManyLeast;  // the workspace is for any window
    most = most < least ? most : least;
    most = most < 1 || !p.many ? 1 : most;
    p.per = (int)((seen + most - 1) / most < kManyLeast ? kManyLeast : (seen + most - 1) / most);
    p.splits = (int)((seen + p.per - 1) / p.per);
    if (p.splits < 1 || !p.many) p.splits = 1;
    p.many_wg = p.many ? wg * p.splits : 0;
    p.many_join = p.splits > 1 ? (rows * nh + kT / (d_head / 8) - 1) / (kT / (d_head / 8)) : 0;
    p.parts = p.few_wg + p.many_wg + p.many_join;
    p.room = p.few_wg + (p.many ? wg * most : 0) + (most > 1 ? (rows * nh + kT / (d_head / 8) - 1) / (kT / (d_head / 8)) : 0);
    const int64_t fs = p.flat ? 2 * kShares * kFew : p.few && p.few_parts > 1 ? p.few_wg * kFew : 0, ms = most > 1 ? most * rows * nh : 0;
    p.words = kCounts * 4;
    p.few_o = (p.words + (1 + p.room) * 4 + 15) & ~(int64_t)15;
    p.few_ml = p.few_o + fs * d_head * 4;
    p.many_o = p.few_ml + fs * 8;
    p.many_ml = p.many_o + ms * d_head * 4;
    p.ws_bytes = p.many_ml + ms * 8;
    return p;
}
}  // namespace

CacheAttnPlan cache_attn_plan(int64_t rows, int nh, int nkv, int d_head, int64_t n_seqs, int64_t max_rows,
                              int64_t max_len) {
    const Plan p = plan_of(rows, nh, nkv, d_head, n_seqs, max_rows, max_len, 0);
    return CacheAttnPlan{p.room, p.ws_bytes};
}

int32_t launch_cache_attention(const uint16_t* q, int64_t ldq, int nh, const CacheView& c, int fmt, int d_head,
                               int64_t max_rows, int64_t window, uint16_t* o, int64_t ldo, const FusedQuant* fq,
                               void* ws, hipStream_t s) {
    const bool quant = fq && fq->q;
    if (window >= (int64_t)1 << 30) window = 0;  // beyond any position: none
    const Plan pl = plan_of(c.rows, nh, c.nkv, d_head, c.n_seqs, max_rows, (int64_t)c.max_pages << c.page_shift, window);
    char* base = (char*)ws;
    uint32_t* words = (uint32_t*)(base + pl.words);
    AttnArgs a;
    a.c = c;
    a.q = q;
    a.ldq = ldq;
    a.nh = nh;
    a.grp = nh / c.nkv;
    a.max_rows = (int)(max_rows < c.rows ? max_rows : c.rows);
    a.window = (int)window;
    a.few_on = pl.few;
    a.splits = pl.splits;
    a.per = pl.per;
    a.flat = pl.flat;
    a.few_parts = pl.few_parts;
    a.counts = (int32_t*)base;
    a.c2 = (float)(1.4426950408889634 / sqrt((double)d_head));
    a.o = o;
    a.ldo = ldo;
    a.pred = quant ? fq->pred : nullptr;
    a.used = quant ? (int32_t*)words : nullptr;
    a.q8 = quant ? fq->q : nullptr;
    a.ldq8 = quant ? fq->ldq : 0;
    a.qfmt = quant ? fq->fmt : FP8_E4M3;
    a.parts = words + 1;
    a.few_o = (float*)(base + pl.few_o);
    a.few_ml = (float2*)(base + pl.few_ml);
    a.many_o = (float*)(base + pl.many_o);
    a.many_ml = (float2*)(base + pl.many_ml);
    a.many_wg = (int)pl.many_wg;
    if (quant && pl.few && (pl.flat || pl.few_parts > 1)) {
        const int n = c.n_seqs * c.nkv;
        hipLaunchKernelGGL(clear_kernel, dim3((unsigned)((n + kT - 1) / kT)), dim3(kT), 0, s, a.counts, n);
    }
    with_cache(fmt, d_head, [&](auto F, auto D) {
        constexpr int kF = decltype(F)::value, kD = decltype(D)::value;
        auto go = [&](auto kernel, int64_t wg) {
            if (wg == 0) return;
            hipLaunchKernelGGL(kernel, dim3((unsigned)wg), dim3(kT), 0, s, a);
            a.parts += wg;
        };
        if (pl.many && pl.few) go(attn_kernel<kF, kD, true, true>, pl.many_wg + pl.few_wg);
        else if (pl.many) go(attn_kernel<kF, kD, true, false>, pl.many_wg);
        else go(attn_kernel<kF, kD, false, true>, pl.few_wg);
        go(many_join_kernel<kD>, pl.many_join);
    });
    int32_t st = hip_status();
    if (st == FP8_OK && quant) {
        const int64_t cols = (int64_t)nh * d_head;
        with_fmt(fq->fmt, [&](auto QF) {
            hipLaunchKernelGGL((quant_finish_kernel<decltype(QF)::value>), dim3((unsigned)(c.rows < 512 ? c.rows : 512)),
                               dim3(kT), 0, s, c, o, cols, ldo, max_rows, fq->margin, words, (int)pl.parts, fq->bias,
                               fq->amax_bits, fq->flags, fq->q, fq->ldq);
        });
        st = hip_status();
    }
    return st;
}

}  // namespace fp8lin
