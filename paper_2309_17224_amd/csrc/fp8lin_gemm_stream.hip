// FP8 matmul for outputs too small to fill the chip with 256 x 256 tiles
// (decode, batched decode, short prompts, small layers), for gfx950.
// C[m, n] = 2^-(ba + bb) * sum_k A[m, k] * B[n, k], K a multiple of 128.
//
// These products are bound by how fast each compute unit can pull operand
// rows into LDS: it keeps about 128 outstanding 128-byte fills, whatever the
// instruction mix, so the time is (rows of the tile) x K per workgroup times
// the rounds of workgroups.  A workgroup therefore takes a small tile of
// 16 MB x 16 NB outputs, chosen so that the grid is one round (or a few whole
// rounds) of the 256 compute units, and its four waves split k, not the tile:
//  * Every stage copies KC bytes of k of the tile's 16 (MB + NB) rows with
//    global_load_lds_dwordx4 (runs of KC contiguous bytes per row), three
//    stages in LDS, two in flight.  Weight rows that no other workgroup reads
//    carry the non-temporal hint.
//  * KC = 512 (up to 96 rows): wave w multiplies the whole tile over the 128
//    bytes of k at 128 w of each stage.  KC = 256 (up to 192 rows): waves w
//    and w + 2 share a 128-byte slice, each half of the tile's columns.  No
//    fragment is read from LDS twice.  KC = 128 (256 rows): the waves take
//    quarters of the tile, and k is not split (512 x 8192 x 8192: 67 us in
//    256-row tiles, 61 in 8 x 4, 48 in 8 x 8).
//  * The partial sums are added through LDS in a fixed order, so the
//    result does not depend on timing.
//  * 16-byte chunk c of LDS row r is stored at chunk c ^ (r % 16): the lanes
//    of every ds_read_b128 phase (see fp8lin_gemm.hip) hit distinct banks.
#include "fp8lin_mm_stream.h"

namespace fp8lin {
namespace {

struct Plain {
    using Args = MmArgs;
    static constexpr bool kPlain = true, kPair = false;
};

template <int FA, int FB, int MB, int NB>
void launch_one(const MmArgs& a, hipStream_t s) {
    const int tm = (int)((a.M + 16 * MB - 1) / (16 * MB)), tn = (int)((a.N + 16 * NB - 1) / (16 * NB));
    hipLaunchKernelGGL((gemm_nt_stream<FA, FB, MB, NB, Plain>), dim3((unsigned)(tm * tn)), dim3(stream_threads(MB)), 0, s,
                       a, tm, tn, tm == 1);
}

template <int FA, int FB>
void launch_t(int mb, int nb, const MmArgs& a, hipStream_t s) {
#define FP8LIN_STREAM_CASE(MB, NB) \
    if (mb == MB && nb == NB) return launch_one<FA, FB, MB, NB>(a, s);
    FP8LIN_STREAM_TILES(FP8LIN_STREAM_CASE)
#undef FP8LIN_STREAM_CASE
}

}  // namespace

// Estimated time (us) of the product with tiles of 16 MB x 16 NB: linear fits
// to 220 shapes x 31 tiles on MI355X (M 1-1500, weights 512-57344 wide), one
// for each kind of tile, which pick a tile within 0.4 % of the best measured
// one on average (12 % at worst, on products of 7 us).
struct StreamFit {
    double launch, round,     // once; per round of workgroups (prologue, epilogue)
        copy, copy_alone,     // MB copied by the busiest compute unit; shared out over its resident workgroups
        stage, mfma,          // its k-bytes of one tile row; its 16 x 16 blocks times k
        weight, weight_part,  // 100 MB of weight; scaled by how much of the last round is empty
        weight_l2, out;       // GB of weight over all rows of tiles; 1e7 outputs
};
constexpr StreamFit kFitDecode{3.479, 0, 2.252, 10.7, 1.913, 0, 0, 6.091, 0, 49.961};   // MB = 1, M <= 16
constexpr StreamFit kFitRows16{1.9, 0.945, 3.85, 16.168, 1.062, 0, 0, 2.467, 0, 13.651};  // MB = 1, M > 16
constexpr StreamFit kFitWide16{2.642, 0.877, 8.195, 0, 9.952, 0, 7.805, 0, 0, 10.343};    // MB = 1, KC = 256
constexpr StreamFit kFit512{2.092, 1.166, 0, 11.704, 2.084, 29.093, 2.814, 1.35, 0, 18.941};
constexpr StreamFit kFit256{2.158, 1.72, 0, 8.853, 5.36, 23.636, 3.739, 1.877, 0, 12.579};
constexpr StreamFit kFit128{2.519, 5.459, 0, 6.509, 0, 35.324, 0, 6.546, 1.301, 6.557};

int64_t stream_workgroups(int64_t M, int64_t N, int mb, int nb) {
    return ((M + 16 * mb - 1) / (16 * mb)) * ((N + 16 * nb - 1) / (16 * nb));
}

// A decode's weight streams through as many workgroups as it takes, and the
// rounds cost nothing but the bytes where each copies for some microseconds.
// With rows as short as these each round past the first adds about this much
// (1 x 57344 x 128: 9.8 us in the 1792 workgroups of 32 columns, 6.7 in 448 of
// 128; 1 x 22016 x 768 7.1 and 5.4 in 230 of 96).
constexpr int64_t kShortK = 2304;
constexpr double kShortRoundUs = 1.0;

template <int MB, int NB>
static double stream_us(int64_t M, int64_t N, int64_t K) {
    constexpr int kc = stream_kc(MB, NB), lds = kSlBuf * 16 * (MB + NB) * kc;
    constexpr int occ = 160 * 1024 / lds < 4 ? 160 * 1024 / lds : 4;
    const StreamFit& f = kc == 128 ? kFit128 : kc == 256 ? (MB == 1 ? kFitWide16 : kFit256)
                         : MB > 1  ? kFit512
                         : M <= 16 ? kFitDecode
                                   : kFitRows16;
    const int64_t tm = (M + 16 * MB - 1) / (16 * MB), tiles = tm * ((N + 16 * NB - 1) / (16 * NB));
    const int64_t rounds = (tiles + 256 * occ - 1) / (256 * occ), per_cu = (tiles + 255) / 256;
    const double cu_k = (double)per_cu * (double)K, mb_copied = cu_k * 16 * (MB + NB) * 1e-6;
    const double weight = (double)N * (double)K * 1e-8;
    const double empty = tiles > 256 * occ ? (double)(rounds * 256 * occ) / (double)tiles : 1.0;
    const double round = &f == &kFitDecode && K <= kShortK ? kShortRoundUs * (double)(rounds - 1) : f.round * (double)rounds;
    return f.launch + round + f.copy * mb_copied + f.copy_alone * mb_copied / (double)(per_cu < occ ? per_cu : occ) +
           f.stage * cu_k * 1e-4 + f.mfma * cu_k * (MB * NB) * 1e-6 + (f.weight + f.weight_part * empty) * weight +
           f.weight_l2 * (double)tm * weight * 0.1 + f.out * (double)M * (double)N * 1e-7;
}

// Every workgroup's fold of its maximum into one word waits for those before
// it, part of which hides behind workgroups that are still multiplying (us).
constexpr double kFoldUs = 0.009;

// The tile with the smallest estimate.  With an epilogue amax, of the tiles
// that sum in the same order (the same KC), so that an output's bits do not
// depend on whether its amax is asked for, the best one with the folds counted
// (256 x 768 x 768 with its amax: 14.4 us in the 768 workgroups that are best
// without, 8.1 in 96; in gemm_nt_256 10.2).
double stream_tile(int64_t M, int64_t N, int64_t K, bool with_amax, int* mb, int* nb, bool even) {
    double best = 0;
    int kc = 0;
#define FP8LIN_STREAM_COST(MB, NB)                                                                             \
    if ((16 * (MB - 1) < M || MB == 1) && (NB % 2 == 0 || !even))                                              \
        if (const double t = stream_us<MB, NB>(M, N, K); best == 0 || t < best) {                              \
            best = t;                                                                                          \
            *mb = MB;                                                                                          \
            *nb = NB;                                                                                          \
            kc = stream_kc(MB, NB);                                                                            \
        }
    FP8LIN_STREAM_TILES(FP8LIN_STREAM_COST)
#undef FP8LIN_STREAM_COST
    if (!with_amax) return best;
    double best_fold = 0;
#define FP8LIN_STREAM_COST(MB, NB)                                                                             \
    if ((16 * (MB - 1) < M || MB == 1) && stream_kc(MB, NB) == kc)                                             \
        if (const double t = stream_us<MB, NB>(M, N, K) + kFoldUs * (double)stream_workgroups(M, N, MB, NB);   \
            best_fold == 0 || t < best_fold) {                                                                 \
            best_fold = t;                                                                                     \
            *mb = MB;                                                                                          \
            *nb = NB;                                                                                          \
        }
    FP8LIN_STREAM_TILES(FP8LIN_STREAM_COST)
#undef FP8LIN_STREAM_COST
    return best;
}

bool stream_tile_at(int i, int* mb, int* nb) {
#define FP8LIN_STREAM_ENTRY(MB, NB) {MB, NB},
    static constexpr int tiles[][2] = {FP8LIN_STREAM_TILES(FP8LIN_STREAM_ENTRY)};
#undef FP8LIN_STREAM_ENTRY
    if (i < 0 || i >= (int)(sizeof(tiles) / sizeof(tiles[0]))) return false;
    *mb = tiles[i][0];
    *nb = tiles[i][1];
    return true;
}

void launch_gemm_stream(int fa, int fb, int mb, int nb, const MmArgs& a, hipStream_t s) {
    if (fa == FP8_E4M3 && fb == FP8_E4M3) launch_t<FP8_E4M3, FP8_E4M3>(mb, nb, a, s);
    else if (fa == FP8_E5M2 && fb == FP8_E4M3) launch_t<FP8_E5M2, FP8_E4M3>(mb, nb, a, s);
    else launch_t<FP8_E4M3, FP8_E5M2>(mb, nb, a, s);
}

}  // namespace fp8lin
