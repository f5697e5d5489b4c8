// The gated feed-forward's two products on 192x256 tiles of the deferred-epilogue kernel (gemm_defer.h): rows, columns and contractions that
// end inside a tile or a stage.
#include <algorithm>
#include "gemm_defer.h"

namespace tweo {

template <int D, int GATE, bool KEEP>
static hipError_t launch_inst(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    using T = DeferTile<3>;
    constexpr auto kernel = gemm_nt_defer_gated_kernel<D, 3, true, GATE, KEEP>;
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

// a tile is written out over the first 15, 7 or 5 stages of the next one, never its last three
template <int GATE, bool KEEP>
static hipError_t launch_stages(const GemmArgs &a, const GatedDev &gd, hipStream_t s)
{
    const int64_t kt = (a.K + 127) / 128;
    if (kt >= 18)
        return launch_inst<15, GATE, KEEP>(a, gd, s);
    return kt >= 10 ? launch_inst<7, GATE, KEEP>(a, gd, s) : launch_inst<5, GATE, KEEP>(a, gd, s);
}

hipError_t launch_defer_any_gated(const GemmArgs &a, bool gelu, const GatedDev &gd, hipStream_t s)
{
    if (gelu)
        return gd.gu != nullptr ? launch_stages<2, true>(a, gd, s) : launch_stages<2, false>(a, gd, s);
    return gd.gu != nullptr ? launch_stages<1, true>(a, gd, s) : launch_stages<1, false>(a, gd, s);
}

}  // namespace tweo
