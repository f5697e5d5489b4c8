// Pieces of the 8-bit casts (gfx950): magnitudes, conversions, the byte transposition of the transposed copies.
#pragma once
#include "device_utils.h"

namespace tweo {

constexpr int kQuantThreads = 256;

__device__ __forceinline__ uint32_t pk_absmax(uint32_t m, uint32_t d)
{
    u16x2 a = __builtin_bit_cast(u16x2, m);
    u16x2 b = __builtin_bit_cast(u16x2, d & 0x7FFF7FFFu);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, b));
}

__device__ __forceinline__ uint32_t pk_absmax4(uint32_t m, uint4 v)
{
    m = pk_absmax(m, v.x);
    m = pk_absmax(m, v.y);
    m = pk_absmax(m, v.z);
    return pk_absmax(m, v.w);
}

__device__ __forceinline__ float sat_e4m3(float v)
{
    float c = __builtin_amdgcn_fmed3f(v, -448.0f, 448.0f);
    return v != v ? v : c;
}

__device__ __forceinline__ uint32_t cvt4_e4m3(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(sat_e4m3(a), sat_e4m3(b), 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(sat_e4m3(c), sat_e4m3(d), r, true);
    return (uint32_t)r;
}

// E5M2, the gradient format of the HYBRID recipe (Sec. 4.3): same cast with the range +-57344.
__device__ __forceinline__ float sat_e5m2(float v)
{
    float c = __builtin_amdgcn_fmed3f(v, -57344.0f, 57344.0f);
    return v != v ? v : c;
}

__device__ __forceinline__ uint32_t cvt4_e5m2(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_bf8_f32(sat_e5m2(a), sat_e5m2(b), 0, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(sat_e5m2(c), sat_e5m2(d), r, true);
    return (uint32_t)r;
}

template <bool E5M2>
__device__ __forceinline__ uint32_t cvt4_f8(float a, float b, float c, float d)
{
    if constexpr (E5M2)
        return cvt4_e5m2(a, b, c, d);
    else
        return cvt4_e4m3(a, b, c, d);
}

template <bool E5M2>
__device__ __forceinline__ float scale_f8(float amax)
{
    return scale_from_amax_range(amax, E5M2 ? 57344.0f : 448.0f);
}

// rows a,b,c,d (one dword = 4 bytes each) -> columns t0..t3 of the 4x4 byte matrix
__device__ __forceinline__ void transpose4x4_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d,
                                                   uint32_t &t0, uint32_t &t1, uint32_t &t2,
                                                   uint32_t &t3)
{
    uint32_t p0 = __builtin_amdgcn_perm(b, a, 0x05010400u);  // a0 b0 a1 b1
    uint32_t p1 = __builtin_amdgcn_perm(b, a, 0x07030602u);  // a2 b2 a3 b3
    uint32_t p2 = __builtin_amdgcn_perm(d, c, 0x05010400u);  // c0 d0 c1 d1
    uint32_t p3 = __builtin_amdgcn_perm(d, c, 0x07030602u);  // c2 d2 c3 d3
    t0 = __builtin_amdgcn_perm(p2, p0, 0x05040100u);         // a0 b0 c0 d0
    t1 = __builtin_amdgcn_perm(p2, p0, 0x07060302u);         // a1 b1 c1 d1
    t2 = __builtin_amdgcn_perm(p3, p1, 0x05040100u);         // a2 b2 c2 d2
    t3 = __builtin_amdgcn_perm(p3, p1, 0x07060302u);         // a3 b3 c3 d3
}

// Delayed scaling (Sec. 4.3: the recipe the paper trained with) hands the cast a scale that was
// fixed before this tensor was seen and wants this tensor's amax back for the history: DELAYED
// kernels read the scale itself from `amax`, and add the maximum magnitude pattern of what they
// load to *amax_acc (one atomicMax per workgroup, skipped when already covered).
template <int WAVES = kQuantThreads / kWave>
__device__ __forceinline__ void quant_amax_commit(uint32_t m, uint32_t *amax_acc)
{
    __shared__ uint32_t red[WAVES];
    uint32_t r = (m & 0xFFFFu) > (m >> 16) ? (m & 0xFFFFu) : (m >> 16);
    r = wave_reduce_max_u32(r);
    if ((threadIdx.x & (kWave - 1)) == 0)
        red[threadIdx.x / kWave] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            r = red[w] > r ? red[w] : r;
        const uint32_t mine = r << 16;
        if (mine > __atomic_load_n(amax_acc, __ATOMIC_RELAXED))
            atomicMax(amax_acc, mine);
    }
}

}  // namespace tweo
