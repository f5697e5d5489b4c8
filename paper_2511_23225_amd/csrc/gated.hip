// Gradients of the gated feed-forward's product h = act(g) * u, cast for the linears' gradients (gfx950):
//
//   dg = bf16(dh * u * act'(g)),  du = bf16(dh * act(g)),  act'(g) = p + g p (1 - p) z'(g)   (activation.h)
//   codes of (dg | du) [M, 2F] with one scale, and their transposed copy
//
// dg and du are formed on the way into both passes (the maximum, the cast) and never stored: 6 bytes are read in each and 4
// written in the second, for 10 written and read again by an activation's gradient in front of a cast.  Under delayed scaling there is
// one pass.
#include <algorithm>
#include "activation.h"
#include "cast.h"
#include "kernels.h"

namespace tweo {

int num_cus_public();

constexpr int kGatedTile = 128;

struct GatedGradDev {
    const uint16_t *dh, *gu;
    int64_t rows, cols;  // M, F
    int64_t tiles_x, tiles;
    GateCoef act;
    float slope0, slope1;  // z'(g) = slope0 + slope1 g^2
    uint8_t *q, *qT;
    const uint32_t *partials;
    int n_partials;
    const float *scale;  // the scale itself, or nullptr: from the partials
    float *scalars;      // where amax, scale and inverse go, or nullptr
    uint32_t *amax_acc;  // delayed scaling: the maximum's word
};

// dg and du of one element
__device__ __forceinline__ void gated_grad_one(float dh, float g, float u, const GatedGradDev &c, float &dg, float &du)
{
    const float p = gate_share(g, c.act), b = __builtin_amdgcn_fmed3f(g, -0x1p60f, 0x1p60f), gp = g * p;
    du = dh * gp;
    dg = dh * u * __builtin_fmaf(gp * (1.0f - p), __builtin_fmaf(c.slope1, b * b, c.slope0), p);
}

__device__ __forceinline__ void gated_grad_vec(uint4 dh, uint4 g, uint4 u, const GatedGradDev &c, uint4 &dg, uint4 &du)
{
    const uint32_t d[4] = {dh.x, dh.y, dh.z, dh.w}, gg[4] = {g.x, g.y, g.z, g.w}, uu[4] = {u.x, u.y, u.z, u.w};
    uint32_t a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float dg0, dg1, du0, du1;
        gated_grad_one(bf16lo_to_f32(d[k]), bf16lo_to_f32(gg[k]), bf16lo_to_f32(uu[k]), c, dg0, du0);
        gated_grad_one(bf16hi_to_f32(d[k]), bf16hi_to_f32(gg[k]), bf16hi_to_f32(uu[k]), c, dg1, du1);
        a[k] = pack_bf16x2(dg0, dg1);
        b[k] = pack_bf16x2(du0, du1);
    }
    dg = make_uint4(a[0], a[1], a[2], a[3]);
    du = make_uint4(b[0], b[1], b[2], b[3]);
}

enum GatedPass { kGatedAmax, kGatedCast, kGatedDelayed };

// A workgroup takes tiles of 128 rows by 128 columns of h, a lane 8x8 elements of one, whose codes of dg and du lie F columns apart.
template <int PASS, bool E5M2>
__global__ __launch_bounds__(kQuantThreads) void gated_grad_kernel(GatedGradDev c)
{
    __shared__ uint4 turned[PASS == kGatedAmax ? 1 : 2 * kGatedTile * kGatedTile / 16];
    __shared__ uint32_t red[kQuantThreads / kWave];
    const int t = threadIdx.x, cg = t & 15, rg = t >> 4;
    const int64_t wide = 2 * c.cols;
    uint32_t mx = 0;
    float scale = 0.0f;
    bool have_scale = PASS == kGatedAmax;
    for (int64_t tile = blockIdx.x; tile < c.tiles; tile += gridDim.x) {
        const int64_t R = tile / c.tiles_x * kGatedTile, C = tile % c.tiles_x * kGatedTile, r0 = R + rg * 8, c0 = C + cg * 8;
        const bool active = r0 < c.rows && c0 < c.cols;  // whole 8x8 blocks: in or out
        const uint16_t *dh = c.dh + (active ? r0 * c.cols + c0 : 0), *g = c.gu + (active ? r0 * wide + c0 : 0);
        uint4 a[8], b[8], d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            d[i] = *(const uint4 *)(dh + i * c.cols);
            a[i] = *(const uint4 *)(g + i * wide);
            b[i] = *(const uint4 *)(g + i * wide + c.cols);
        }
        if (!have_scale) {  // behind the first loads, so that the latencies overlap
            have_scale = true;
            if (c.scale != nullptr) {
                scale = *c.scale;
            } else {
                uint32_t m = 0;
                for (int i = t; i < c.n_partials; i += kQuantThreads)
                    m = max(m, c.partials[i]);
                m = wave_reduce_max_u32(m);
                if ((t & (kWave - 1)) == 0)
                    red[t / kWave] = m;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kQuantThreads / kWave; ++w)
                    m = max(m, red[w]);
                scale = scale_f8<E5M2>(bits_to_f32(m));
                if (blockIdx.x == 0 && t == 0) {
                    c.scalars[0] = bits_to_f32(m);
                    c.scalars[1] = scale;
                    c.scalars[2] = 1.0f / scale;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            gated_grad_vec(d[i], a[i], b[i], c, a[i], b[i]);
        if constexpr (PASS != kGatedCast) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                m = pk_absmax4(pk_absmax4(m, a[i]), b[i]);
            mx = active ? pk_absmax(m, mx) : mx;
        }
        if constexpr (PASS != kGatedAmax) {
            if (tile != (int64_t)blockIdx.x)
                __syncthreads();  // the tile before has been read
            uint8_t *q = c.q + (active ? r0 * wide + c0 : 0);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t lo[8], hi[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4 v = half ? b[i] : a[i];
                    lo[i] = cvt4_f8<E5M2>(bf16lo_to_f32(v.x) * scale, bf16hi_to_f32(v.x) * scale, bf16lo_to_f32(v.y) * scale, bf16hi_to_f32(v.y) * scale);
                    hi[i] = cvt4_f8<E5M2>(bf16lo_to_f32(v.z) * scale, bf16hi_to_f32(v.z) * scale, bf16lo_to_f32(v.w) * scale, bf16hi_to_f32(v.w) * scale);
                    if (active)
                        *(uint2 *)(q + i * wide + half * c.cols) = make_uint2(lo[i], hi[i]);
                }
                uint32_t ta[8], tb[8];  // column j of the block: rows 0-3, rows 4-7
                transpose4x4_bytes(lo[0], lo[1], lo[2], lo[3], ta[0], ta[1], ta[2], ta[3]);
                transpose4x4_bytes(hi[0], hi[1], hi[2], hi[3], ta[4], ta[5], ta[6], ta[7]);
                transpose4x4_bytes(lo[4], lo[5], lo[6], lo[7], tb[0], tb[1], tb[2], tb[3]);
                transpose4x4_bytes(hi[4], hi[5], hi[6], hi[7], tb[4], tb[5], tb[6], tb[7]);
                uint8_t *w = (uint8_t *)turned + half * kGatedTile * kGatedTile + cg * 8 * kGatedTile + (((rg >> 1) ^ (cg & 7)) << 4) + (rg & 1) * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *(uint2 *)(w + j * kGatedTile) = make_uint2(ta[j], tb[j]);
            }
            __syncthreads();
            const int piece = t & 7;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int half = i >> 2, col = (t >> 3) + 32 * (i & 3);
                const v4i v = __builtin_bit_cast(v4i, turned[half * (kGatedTile * kGatedTile / 16) + col * (kGatedTile / 16) + (piece ^ ((col >> 3) & 7))]);
                if (C + col < c.cols && R + piece * 16 < c.rows)
                    *(v4i *)(c.qT + (half * c.cols + C + col) * c.rows + R + piece * 16) = v;
            }
        }
    }
    if constexpr (PASS == kGatedAmax) {
        uint32_t r = max(mx & 0xFFFFu, mx >> 16);
        r = wave_reduce_max_u32(r);
        if ((t & (kWave - 1)) == 0)
            red[t / kWave] = r;
        __syncthreads();
        if (t == 0) {
#pragma unroll
            for (int w = 1; w < kQuantThreads / kWave; ++w)
                r = max(r, red[w]);
            const_cast<uint32_t *>(c.partials)[blockIdx.x] = r << 16;
        }
    }
    if constexpr (PASS == kGatedDelayed)
        quant_amax_commit(mx, c.amax_acc);
}

template <bool E5M2>
static hipError_t launch_grad(const GatedGradCall &call, GatedGradDev c, hipStream_t s)
{
    const unsigned tiles = (unsigned)c.tiles;
    // each workgroup ends in a word of its own, or in an atomic: three a CU walk the tiles
    const unsigned few = (unsigned)std::min<int64_t>({(int64_t)c.tiles, 3 * (int64_t)num_cus_public(), kGatedPartials});
    float *state = (float *)call.state;
    if (state != nullptr && !call.bootstrap) {
        c.scale = state + 17;
        c.amax_acc = (uint32_t *)state + 16;
        hipLaunchKernelGGL((gated_grad_kernel<kGatedDelayed, E5M2>), dim3(few), dim3(kQuantThreads), 0, s, c);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? launch_delayed_update(state, false, E5M2, nullptr, 0, call.scalars, s) : e;
    }
    c.partials = call.partials;
    c.n_partials = (int)few;
    hipLaunchKernelGGL((gated_grad_kernel<kGatedAmax, false>), dim3(few), dim3(kQuantThreads), 0, s, c);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && state != nullptr) {
        e = launch_delayed_update(state, true, E5M2, call.partials, (int)few, call.scalars, s);
        c.scale = state + 21;
    }
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((gated_grad_kernel<kGatedCast, E5M2>), dim3(tiles), dim3(kQuantThreads), 0, s, c);
    return hipGetLastError();
}

hipError_t launch_gated_grad(const GatedGradCall &call, hipStream_t s)
{
    GatedGradDev c{};
    c.dh = (const uint16_t *)call.dh;
    c.gu = (const uint16_t *)call.gu;
    c.rows = call.M;
    c.cols = call.F;
    c.tiles_x = (call.F + kGatedTile - 1) / kGatedTile;
    c.tiles = c.tiles_x * ((call.M + kGatedTile - 1) / kGatedTile);
    c.act = gate_coef(call.gelu);
    constexpr double k = 1.5957691216057307118;  // 2 sqrt(2 / pi)
    c.slope0 = call.gelu ? (float)k : 1.0f;
    c.slope1 = call.gelu ? (float)(3 * k * 0.044715) : 0.0f;
    c.q = call.q;
    c.qT = call.qT;
    c.scalars = call.scalars;
    return call.e5m2 ? launch_grad<true>(call, c, s) : launch_grad<false>(call, c, s);
}

}  // namespace tweo
