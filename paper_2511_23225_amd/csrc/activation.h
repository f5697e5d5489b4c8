// The gate's activations: act(g) = g * p, p = sigmoid(z), with z = g (SiLU) or 2 sqrt(2/pi) (g + 0.044715 g^3) (GELU, tanh form).
#pragma once
#include "device_utils.h"
#include "kernels.h"

namespace tweo {

// z in units of log 2 is g * (c0 + c1 g^2): one formula for both, c1 = 0 for SiLU.
static inline GateCoef gate_coef(bool gelu)
{
    constexpr double log2e = 1.4426950408889634074, k = 1.5957691216057307118;  // 2 sqrt(2 / pi)
    return gelu ? GateCoef{(float)(k * log2e), (float)(k * 0.044715 * log2e)} : GateCoef{(float)log2e, 0.0f};
}

// z is within e |z| of itself: e = 2^-23 for SiLU (the constant's rounding and the product's), 2^-22 for GELU (those of both constants, the square, the
// sum and the product).  The base-2 exponential and the reciprocal are the hardware's, 1 step each, so p is within e |z| + 2^-21 of
// itself.  A g that would square to infinity (0 times that is NaN) counts as 2^60.  Below p = 2^-128 (g under -88) p is 0.
__device__ __forceinline__ float gate_share(float g, const GateCoef &c)
{
    const float b = __builtin_amdgcn_fmed3f(g, -0x1p60f, 0x1p60f);
    const float z = b * __builtin_fmaf(c.c1, b * b, c.c0);
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-z));
}

// The exponential of it by itself, p = 1 / (1 + this): the same bits
template <bool GELU>
__device__ __forceinline__ float gate_exp(float g, const GateCoef &c)
{
    if constexpr (GELU) {
        const float b = __builtin_amdgcn_fmed3f(g, -0x1p60f, 0x1p60f);
        return __builtin_amdgcn_exp2f(-(b * __builtin_fmaf(c.c1, b * b, c.c0)));
    }
    return __builtin_amdgcn_exp2f(-(g * c.c0));
}

// The share with the sum's rounding and the reciprocal's taken back, where memory leaves time for it: p is within (e |z| + 2^-22) (1 - p) and the
// half step of its own rounding, 2^-24, of itself.
// (Beyond what the reciprocal of a number gives the correction is not one, and times 0.)
template <bool GELU>
__device__ __forceinline__ float gate_share_near(float g, const GateCoef &c)
{
    const float e = gate_exp<GELU>(g, c), d = 1.0f + e, p = __builtin_amdgcn_rcpf(d);
    const float r = __builtin_fmaf(-(e - (d - 1.0f)), p, __builtin_fmaf(-d, p, 1.0f));
    return __builtin_fmaf(p, __builtin_amdgcn_fmed3f(r, -0x1p-20f, 0x1p-20f), p);
}

__device__ __forceinline__ float gated(float g, float u, const GateCoef &c) { return g * gate_share(g, c) * u; }

}  // namespace tweo
