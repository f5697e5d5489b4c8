// Launches of the gated feed-forward's two products (gemm_gated.h): on the deferred-epilogue kernel (gemm_defer.h, GATE) where there are
// tiles and stages enough, else on the ring kernel's tiles (gemm_ring.h).
#include <algorithm>
#include <cmath>
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
    const GemmDev g = gemm_dev(a, T::BM, T::BN / 2);
    launch_gemm_kernel(kernel, dim3((unsigned)(g.tiles_m * g.tiles_n)), dim3(T::THREADS), T::LDS_BYTES, s, g, gd);
    return hipGetLastError();
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

static int pick_shape(int64_t M, int64_t F, int64_t K, bool int8)
{
    const int64_t tiles = ((M + 63) / 64) * ((F + 31) / 32);
    const int forced = gemm_tile_override();
    for (int i = 0; forced != 0 && i < kGatedShapes; ++i) {
        static const int variant[kGatedShapes] = {4, 18, 19, 20, 21, 15, 24};
        if (variant[i] == forced && shape_fits(i, M, F, K, int8))
            return i;
    }
    if (tiles <= num_cus_public())
        return kGated64x64g2;
    if (M <= 64 || tiles <= 2 * num_cus_public())
        return kGated64x64;
    return kGated128x128x2;
}

hipError_t launch_fp8_gated(const GemmArgs &a, bool gelu, void *gu, hipStream_t s)
{
    const GatedDev gd{(uint16_t *)gu, gate_coef(gelu)};
    const int shape = pick_shape(a.M, a.N, a.K, false);
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
    return launch_ring_shape<true>(a, GatedDev{nullptr, gate_coef(gelu)}, pick_shape(a.M, a.N, a.K, true), s);
}

}  // namespace tweo
