// Launches of the gated feed-forward's two products (gemm_gated.h): on the deferred-epilogue kernel (gemm_defer.h, GATE) where there are
// tiles and stages enough, else on the ring kernel's tiles (gemm_ring.h).
#include <algorithm>
#include "gemm_defer.h"
#include "gemm_ring.h"

namespace tweo {

int num_cus_public();

// tiles of M rows by 2F rows of the weight
typedef TileR<64, 64, 2, 2, 1, 4> G64x64;
typedef TileR<64, 64, 2, 2, 2, 8> G64x64g2;
typedef TileR<64, 128, 2, 2, 1, 3> G64x128;
typedef TileR<64, 128, 2, 2, 2, 6> G64x128g2;
typedef TileR<128, 128, 2, 2, 1, 2> G128x128x2;

enum GatedShape { kGated64x64, kGated64x64g2, kGated64x128, kGated64x128g2, kGated128x128x2, kGated256, kGated192, kGatedShapes };
static const int kGatedVariant[kGatedShapes] = {4, 18, 19, 20, 21, 15, 24};  // as tweo_set_gemm_tile counts them

int gated_workgroups(int64_t M, int64_t F, int bm)
{
    return (int)std::min<int64_t>(num_cus_public(), ((M + bm - 1) / bm) * ((F + 127) / 128));
}

template <typename T, bool INT8, bool RAGGED>
static hipError_t launch_inst(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    constexpr auto kernel = gemm_nt_ring_gated_kernel<T, INT8, RAGGED>;
    static bool done = false;
    if (!done) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
        if (e != hipSuccess)
            return e;
        done = true;
    }
    // A launch holds less than 2^32 threads: rows beyond that (2^30 under 8 columns are 2^24 tiles of 64) go into launches of their own.
    constexpr int64_t most = (((int64_t)1 << 32) - 1) / T::THREADS;
    const int64_t tiles_n = (a.N + T::BN / 2 - 1) / (T::BN / 2), rows = std::max<int64_t>(1, most / tiles_n) * T::BM;
    for (int64_t m = 0; m < a.M; m += rows) {
        GemmArgs part = a;
        part.M = std::min(rows, a.M - m);
        part.A += m * a.K;
        part.out = (uint8_t *)a.out + m * a.N * (INT8 && a.out_i8 ? 1 : 2);
        if (INT8)
            part.row_step += m * a.row_step_stride;
        const GatedDev keep{gd.gu != nullptr ? gd.gu + 2 * m * a.N : nullptr, gd.act};
        const GemmDev g = gemm_dev(part, T::BM, T::BN / 2);
        launch_gemm_kernel(kernel, dim3((unsigned)(g.tiles_m * g.tiles_n)), dim3(T::THREADS), T::LDS_BYTES, s, g, keep);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

template <typename T, bool INT8>
static hipError_t launch_shape(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    return a.K % T::BK != 0 ? launch_inst<T, INT8, true>(a, gd, s) : launch_inst<T, INT8, false>(a, gd, s);
}

template <bool INT8>
static hipError_t launch_ring_shape(const GemmArgs &a, const GatedDev &gd, int shape, hipStream_t s)
{
    switch (shape) {
    case kGated64x64: return launch_shape<G64x64, INT8>(a, gd, s);
    case kGated64x64g2: return launch_shape<G64x64g2, INT8>(a, gd, s);
    case kGated64x128: return launch_shape<G64x128, INT8>(a, gd, s);
    case kGated64x128g2: return launch_shape<G64x128g2, INT8>(a, gd, s);
    default: return launch_shape<G128x128x2, INT8>(a, gd, s);
    }
}

template <int D, int GATE, bool KEEP>
static hipError_t launch_defer_inst(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    using T = DeferTile<4>;
    constexpr auto kernel = gemm_nt_defer_gated_kernel<D, 4, false, GATE, KEEP>;
    static bool done = false;
    if (!done) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
        if (e != hipSuccess)
            return e;
        done = true;
    }
    launch_gemm_kernel(kernel, dim3((unsigned)gated_workgroups(a.M, a.N, T::BM)), dim3(T::THREADS), T::LDS_BYTES, s, gemm_dev(a, T::BM, T::BN / 2), gd);
    return hipGetLastError();
}

// a tile is written out over the first 15, 7 or 5 stages of the next one, never its last
template <int GATE, bool KEEP>
static hipError_t launch_defer(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    const int64_t kt = a.K / 128;
    if (kt >= 16)
        return launch_defer_inst<15, GATE, KEEP>(a, gd, s);
    return kt >= 8 ? launch_defer_inst<7, GATE, KEEP>(a, gd, s) : launch_defer_inst<5, GATE, KEEP>(a, gd, s);
}

static bool shape_fits(int shape, int64_t M, int64_t F, int64_t K, bool int8)
{
    constexpr int64_t kMax = (int64_t)1 << 22;  // 32-bit offsets of a tile's rows
    if (shape == kGated256)
        return !int8 && M % 256 == 0 && F % 128 == 0 && K % 128 == 0 && K >= 6 * 128 && F <= kMax && K <= kMax;
    if (shape == kGated192)
        return !int8 && K > 7 * 128 && F <= kMax && K <= kMax;
    return true;
}

// Per shape, us: a launch; a 128-byte stage with one workgroup on a CU and with two; the end of a round (its epilogue and the next
// tile's first operands), more with both projections stored; how much longer a stage of rows takes that are no whole lines, no whole halves of
// them; TB/s at which operands and results move at best, and the weights under one row of tiles (0.036 a workgroup).  Fitted to 420 shapes of 1 to 16384 rows, 128 to 14336 columns and contractions of
// 128 to 8192, operands cold (10 % rms; the choice costs 1.8 % against the fastest in the geometric mean, 22 % at worst).  What it
// decides, us: 1x5632 under 2048 6.3 on 64x64 tiles in two groups and 9.1 on 64x128; 512x2048 under 768 6.5 and 6.1; 926x7680 under 256 25.6
// on 64x64 tiles and 17.0 on 128x128; 1395x9248 under 3616 156 on 128x128 tiles and 118 on 192x256; 768x9728 under 5632 98, 106 and on whole
// 256x256 tiles 69.  INT8: 64x11008 under 4096 24.3 on 64x64 tiles and 21.8 on 64x128 in two groups, 256 rows 51 and on 128x128 42.
struct GatedRate {
    int bm, bn, per_cu;
    double launch, one, two, round, keep, halves, pieces, tb, stream;
};
static const GatedRate kFp8Rates[kGatedShapes] = {
    {64, 64, 2, 2.3, 0.144, 0.380, 1.3, 0.3, 1.17, 1.28, 5.1, 4.8},   {64, 64, 1, 2.0, 0.121, 0.217, 1.7, 0.3, 1.21, 1.35, 5.2, 6.0},
    {64, 128, 2, 1.7, 0.266, 0.601, 1.8, 0.2, 1.13, 1.32, 3.75, 5.0}, {64, 128, 1, 1.3, 0.239, 0.338, 2.4, 0.3, 1.21, 1.39, 4.1, 5.3},
    {128, 128, 2, 0.9, 0.596, 1.027, 2.5, 0.0, 1.08, 1.20, 2.9, 3.5}, {256, 256, 1, 0.5, 1.071, 1.071, 7.2, 0.0, 1.0, 1.0, 3.3, 3.3},
    {192, 256, 1, 0.5, 0.889, 0.889, 5.3, 0.0, 1.0, 1.23, 4.5, 4.5},
};
static const GatedRate kInt8Rates[kGatedShapes] = {
    {64, 64, 2, 2.2, 0.176, 0.394, 1.6, 0.0, 1.30, 1.27, 4.7, 5.2},   {64, 64, 1, 1.8, 0.158, 0.229, 2.1, 0.0, 1.30, 1.31, 4.45, 5.6},
    {64, 128, 2, 1.7, 0.269, 0.616, 2.4, 0.0, 1.38, 1.40, 4.4, 5.35},  {64, 128, 1, 1.5, 0.239, 0.345, 2.9, 0.0, 1.48, 1.57, 4.6, 5.8},
    {128, 128, 2, 0.9, 0.553, 1.010, 3.5, 0.0, 1.14, 1.27, 2.65, 3.5}, {}, {},
};

static int pick_shape(int64_t M, int64_t F, int64_t K, bool int8, bool keep)
{
    const int64_t cus = num_cus_public(), kt = (K + 127) / 128;
    const int forced = gemm_tile_override();
    int best = kGated64x64;
    double least = 1e300;
    for (int i = 0; i < kGatedShapes; ++i) {
        if (!shape_fits(i, M, F, K, int8))
            continue;
        if (kGatedVariant[i] == forced)
            return i;
        const GatedRate &r = (int8 ? kInt8Rates : kFp8Rates)[i];
        const int64_t tiles = ((M + r.bm - 1) / r.bm) * ((2 * F + r.bn - 1) / r.bn), slots = r.per_cu * cus;
        const double rounds = (double)((tiles + slots - 1) / slots), ragged = K % 128 == 0 ? 1.0 : K % 64 == 0 ? r.halves : r.pieces;
        const double mb = ((double)M * K + 2.0 * F * K + 2.0 * M * F * (keep ? 3 : 1)) * 1e-6;
        const double us = std::max(r.launch + rounds * ((tiles <= cus ? r.one : r.two) * ragged * kt + r.round + (keep ? r.keep : 0.0)), 3.0 + mb / (M <= r.bm ? std::min(r.stream, 0.036 * (double)tiles) : r.tb));
        if (us < least) {
            least = us;
            best = i;
        }
    }
    return best;
}

int fp8_gated_variant(int64_t M, int64_t F, int64_t K, bool keep) { return kGatedVariant[pick_shape(M, F, K, false, keep)]; }

hipError_t launch_fp8_gated(const GemmArgs &a, bool gelu, void *gu, hipStream_t s)
{
    const GatedDev gd{(uint16_t *)gu, gate_coef(gelu)};
    const int shape = pick_shape(a.M, a.N, a.K, false, gu != nullptr);
    if (shape == kGated192)
        return launch_defer_any_gated(a, gelu, gd, s);
    if (shape != kGated256)
        return launch_ring_shape<false>(a, gd, shape, s);
    if (gelu)
        return gu != nullptr ? launch_defer<2, true>(a, gd, s) : launch_defer<2, false>(a, gd, s);
    return gu != nullptr ? launch_defer<1, true>(a, gd, s) : launch_defer<1, false>(a, gd, s);
}

hipError_t launch_i8_gated(const GemmArgs &a, bool gelu, hipStream_t s)
{
    return launch_ring_shape<true>(a, GatedDev{nullptr, gate_coef(gelu)}, pick_shape(a.M, a.N, a.K, true, false), s);
}

}  // namespace tweo
