// Arithmetic that the LayerNorm kernels share: the normalised value in fp64, rounded once to bf16.
#pragma once
#include "device_utils.h"

namespace tweo {

// fp64 -> fp32 such that rounding the result to bf16 (round to nearest even) is the single correct
// rounding of the fp64 value: the 29 mantissa bits that fp32 cannot hold are cut off and, if any
// was set, the last bit that fp32 does hold is set ("round to odd"); the conversion is then exact,
// and a value rounded to odd at 24 bits rounds to 8 bits like the original.  (Below the smallest
// normal fp32, 1.2e-38, the conversion itself rounds again; a normalised activation is either an
// exact zero or many orders of magnitude above that.)
__device__ __forceinline__ float f64_to_f32_for_bf16(double v)
{
    uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)b, cut = lo & 0x1FFFFFFFu;
    const uint32_t lo2 = (lo & 0xE0000000u) | ((cut + 0x1FFFFFFFu) & 0x20000000u);
    b = (b & 0xFFFFFFFF00000000ull) | lo2;
    return (float)__builtin_bit_cast(double, b);
}

// N elements of a row: y = (x - mean) * (rstd * gamma) + beta in fp64 (one rounding more or
// less than the textbook order of operations: 1e-16 relative, far below anything a bf16 rounding
// sees), as packed bf16 pairs.  g / b: the columns' parameters, widened by the caller.
// The way to bf16 goes through the nearest fp32: rounding twice differs from rounding once only if
// the fp32 value is exactly half way between two bf16 values (low half 0x8000), which one element
// in 65536 is; a vector that holds one (and then the wave, once in about 130 vectors) is rounded
// again through the round-to-odd fp32.  Four integer operations per element fewer than that way
// for all (16384x2048: cast 34.4 -> 33.0 us).
// APART holds the second rounding behind its branch, of which the compiler computes parts in front for the longer pieces
// (the forward to bf16 of 16384x2048 46.9 us, 45.2).
template <int N, bool APART = false, typename Param>
__device__ __forceinline__ void ln_pairs(const uint32_t (&x)[N / 2], double mean, double rstd, const Param (&g)[N], const Param (&b)[N],
                                         bool has_beta, uint32_t (&r)[N / 2])
{
    double y[N];
    u16x2 tie = {0xFFFF, 0xFFFF};
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        const double d0 = (double)bf16lo_to_f32(x[k]) - mean, d1 = (double)bf16hi_to_f32(x[k]) - mean;
        const double a0 = rstd * (double)g[2 * k], a1 = rstd * (double)g[2 * k + 1];
        // without a beta nothing is added, so that a zero keeps the sign the product gives it
        y[2 * k] = has_beta ? __builtin_fma(d0, a0, (double)b[2 * k]) : d0 * a0;
        y[2 * k + 1] = has_beta ? __builtin_fma(d1, a1, (double)b[2 * k + 1]) : d1 * a1;
        const float f0 = (float)y[2 * k], f1 = (float)y[2 * k + 1];
        const uint32_t low = __builtin_amdgcn_perm(f32_to_bits(f1), f32_to_bits(f0), 0x05040100u) ^ 0x80008000u;
        tie = __builtin_elementwise_min(tie, __builtin_bit_cast(u16x2, low));
        r[k] = pack_bf16x2(f0, f1);
    }
    if (tie[0] == 0 || tie[1] == 0) {
        if constexpr (APART)
#pragma unroll
            for (int k = 0; k < N; ++k)
                asm volatile("" : "+v"(y[k]));
#pragma unroll
        for (int k = 0; k < N / 2; ++k)
            r[k] = pack_bf16x2(f64_to_f32_for_bf16(y[2 * k]), f64_to_f32_for_bf16(y[2 * k + 1]));
    }
}

// Sum over a wave without LDS: DPP row shifts, then the two row broadcasts (every lane gets it; a shuffle through the
// LDS takes ten times as long, and these sums are a chain in the middle of a row).
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_add_f64(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROW_MASK, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROW_MASK, 0xF, false);
    return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ double wave_sum_f64(double v)
{
    v = dpp_add_f64<0x111, 0xF>(v);
    v = dpp_add_f64<0x112, 0xF>(v);
    v = dpp_add_f64<0x114, 0xF>(v);
    v = dpp_add_f64<0x118, 0xF>(v);
    v = dpp_add_f64<0x142, 0xA>(v);
    v = dpp_add_f64<0x143, 0xC>(v);
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

}  // namespace tweo
