// Launches of the gated feed-forward's two products (gemm_gated.h) on the ring kernel's tiles (gemm_ring.h).
#include <algorithm>
#include "gemm_ring.h"

namespace tweo {

int num_cus_public();

typedef TileR<64, 64, 2, 2, 1, 4> G64x64;
typedef TileR<64, 64, 2, 2, 2, 8> G64x64g2;
typedef TileR<128, 128, 2, 2, 1, 2> G128x128x2;

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
    GemmDev g = gemm_dev(a, T::BM, T::BN / 2);
    launch_gemm_kernel(kernel, dim3((unsigned)((int64_t)g.tiles_m * g.tiles_n)), dim3(T::THREADS), T::LDS_BYTES, s, g, gd);
    return hipGetLastError();
}

template <typename T, bool INT8>
static hipError_t launch_shape(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    return a.K % T::BK != 0 ? launch_inst<T, INT8, true>(a, gd, s) : launch_inst<T, INT8, false>(a, gd, s);
}

template <bool INT8>
static hipError_t launch_gated(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    const int64_t tiles = ((a.M + 63) / 64) * ((a.N + 31) / 32);
    if (tiles <= num_cus_public())
        return launch_shape<G64x64g2, INT8>(a, gd, s);
    if (a.M <= 64 || tiles <= 2 * num_cus_public())
        return launch_shape<G64x64, INT8>(a, gd, s);
    return launch_shape<G128x128x2, INT8>(a, gd, s);
}

hipError_t launch_fp8_gated(const GemmArgs &a, bool gelu, void *gu, hipStream_t s)
{
    return launch_gated<false>(a, GatedDev{(uint16_t *)gu, gate_coef(gelu)}, s);
}

hipError_t launch_i8_gated(const GemmArgs &a, bool gelu, hipStream_t s)
{
    return launch_gated<true>(a, GatedDev{nullptr, gate_coef(gelu)}, s);
}

}  // namespace tweo
