// Gradients of the gated feed-forward's product h = act(g) * u, cast for the linears' gradients (gfx950):
//
//   dg = bf16(dh * u * act'(g)),  du = bf16(dh * act(g)),  act'(g) = p + g p (1 - p) z'(g)   (activation.h)
//   codes of (dg | du) [M, 2F] with one scale, and their transposed copy
//
// dg and du are formed on the way into both passes (the maximum, the cast) and never stored: 6 bytes are read in each and 4
// written in the second, for 10 written and read again by an activation's gradient in front of a cast.  Under delayed scaling there is
// one pass.  Memory bounds both: 16384x5632 97 us (5.7 TB/s) and 175 (5.3 TB/s).
#include <algorithm>
#include "activation.h"
#include "cast.h"
#include "kernels.h"

namespace tweo {

int num_cus_public();

constexpr int kGatedTile = 128, kGatedCols = 4;

struct GatedGradDev {
    const uint16_t *dh, *gu;
    int64_t rows, cols;  // M, F
    int64_t tiles_x, tiles;
    GateCoef act;
    float slope0, slope1;  // GELU: z'(g) = slope0 + slope1 g^2
    uint8_t *q, *qT;
    const uint32_t *partials;
    int n_partials;
    const float *scale;  // the scale itself, or nullptr: from the partials
    float *scalars;      // where amax, scale and inverse go, or nullptr
    uint32_t *amax_acc;  // delayed scaling: the maximum's word
};

// dg and du of one element
template <bool GELU>
__device__ __forceinline__ void gated_grad_one(float dh, float g, float u, const GatedGradDev &c, float &dg, float &du)
{
    const float p = gate_share_near<GELU>(g, c.act), gp = g * p, bend = gp * (1.0f - p);
    du = dh * gp;
    if constexpr (GELU) {
        const float b = __builtin_amdgcn_fmed3f(g, -0x1p60f, 0x1p60f);
        dg = dh * u * __builtin_fmaf(bend, __builtin_fmaf(c.slope1, b * b, c.slope0), p);
    } else {
        dg = dh * u * (p + bend);
    }
}

// W elements (a pair a word): g becomes dg, u du
template <int N>
struct Words {
    uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(const uint16_t *p)
{
    static_assert(N == 2 || N == 4, "8 or 16 bytes");
    Words<N> r;
    if constexpr (N == 4) {
        const uint4 v = *(const uint4 *)p;
        r = {{v.x, v.y, v.z, v.w}};
    } else {
        const uint2 v = *(const uint2 *)p;
        r = {{v.x, v.y}};
    }
    return r;
}
template <bool GELU, int N>
__device__ __forceinline__ void gated_grad_words(const Words<N> &dh, Words<N> &g, Words<N> &u, const GatedGradDev &c)
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float dg0, dg1, du0, du1;
        gated_grad_one<GELU>(bf16lo_to_f32(dh.w[k]), bf16lo_to_f32(g.w[k]), bf16lo_to_f32(u.w[k]), c, dg0, du0);
        gated_grad_one<GELU>(bf16hi_to_f32(dh.w[k]), bf16hi_to_f32(g.w[k]), bf16hi_to_f32(u.w[k]), c, dg1, du1);
        g.w[k] = pack_bf16x2(dg0, dg1);
        u.w[k] = pack_bf16x2(du0, du1);
    }
}

enum GatedPass { kGatedAmax, kGatedCast, kGatedDelayed };

// rows of a tile and threads of its workgroup
constexpr int gated_rows(int pass, bool small) { return !small ? 128 : pass == kGatedAmax ? 32 : 64; }
constexpr int gated_threads(int pass, bool small) { return kGatedTile / kGatedCols * (gated_rows(pass, small) / (small && pass == kGatedAmax ? 2 : 8)); }

// A workgroup takes tiles of 128 rows by 128 columns of h, a lane 8 rows by 4 columns of one, whose codes of dg and du lie F columns apart.
// (Lanes of 8 by 8, 16-byte loads, have half the waves a SIMD: 16384x5632 both passes 10 us more.)
// SMALL: tiles for fewer than two workgroups a CU.  The maximum takes 32 rows at a time (2 a lane), the cast 64 (half as many lanes), whose pieces of
// the transposed copy are half lines.  1024x2048, 128 tiles of 128 rows: 6.2 and 10.1 us, now 5.1 and 9.2.  The one pass under delayed scaling takes 128
// rows whatever the size (there, with the state's update, 13.3 us a call; maximum and cast 13.4).
template <int PASS, bool E5M2, bool SMALL, bool GELU>
__global__ __launch_bounds__(gated_threads(PASS, SMALL)) void gated_grad_kernel(GatedGradDev c)
{
    constexpr int THREADS = gated_threads(PASS, SMALL), W = kGatedCols, ACROSS = kGatedTile / W, N = W / 2, WAVES = THREADS / kWave;
    constexpr int ROWS = SMALL && PASS == kGatedAmax ? 2 : 8, TILE_ROWS = gated_rows(PASS, SMALL), PIECES = TILE_ROWS / 16;
    static_assert(THREADS == TILE_ROWS / ROWS * ACROSS, "a lane's block");
    __shared__ uint4 turned[PASS == kGatedAmax ? 1 : 2 * kGatedTile * PIECES];
    __shared__ uint32_t red[WAVES];
    const int t = threadIdx.x, cg = t % ACROSS, rg = t / ACROSS;
    const int64_t wide = 2 * c.cols;
    uint32_t mx = 0;
    float scale = 0.0f;
    bool have_scale = PASS == kGatedAmax;
    for (int64_t tile = blockIdx.x; tile < c.tiles; tile += gridDim.x) {
        // the cast goes the other way: what the first pass read last may still be in the memory-side cache (16384x5632 both passes
        // 290 us, 280)
        const int64_t id = PASS == kGatedCast ? c.tiles - 1 - tile : tile;
        const int64_t R = id / c.tiles_x * TILE_ROWS, C = id % c.tiles_x * kGatedTile, r0 = R + rg * ROWS, c0 = C + cg * W;
        const bool active = r0 < c.rows && c0 < c.cols;  // whole blocks: in or out
        const uint16_t *dh = c.dh + (active ? r0 * c.cols + c0 : 0), *g = c.gu + (active ? r0 * wide + c0 : 0);
        Words<N> a[ROWS], b[ROWS], d[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            d[i] = load_words<N>(dh + i * c.cols);
            a[i] = load_words<N>(g + i * wide);
            b[i] = load_words<N>(g + i * wide + c.cols);
        }
        if (!have_scale) {  // behind the first loads, so that the latencies overlap
            have_scale = true;
            if (c.scale != nullptr) {
                scale = *c.scale;
            } else {
                uint32_t m = 0;
                for (int i = t; i < c.n_partials; i += THREADS)
                    m = max(m, c.partials[i]);
                m = wave_reduce_max_u32(m);
                if ((t & (kWave - 1)) == 0)
                    red[t / kWave] = m;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WAVES; ++w)
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
        for (int i = 0; i < ROWS; ++i)
            gated_grad_words<GELU>(d[i], a[i], b[i], c);
        if constexpr (PASS != kGatedCast) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    m = pk_absmax(pk_absmax(m, a[i].w[k]), b[i].w[k]);
            mx = active ? pk_absmax(m, mx) : mx;
        }
        if constexpr (PASS != kGatedAmax) {
            if (tile != (int64_t)blockIdx.x)
                __syncthreads();  // the tile before has been read
            uint8_t *q = c.q + (active ? r0 * wide + c0 : 0);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t code[N / 2][8];  // four columns each, by rows
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const Words<N> &v = half ? b[i] : a[i];
#pragma unroll
                    for (int k = 0; k < N / 2; ++k)
                        code[k][i] = cvt4_f8<E5M2>(bf16lo_to_f32(v.w[2 * k]) * scale, bf16hi_to_f32(v.w[2 * k]) * scale,
                                                   bf16lo_to_f32(v.w[2 * k + 1]) * scale, bf16hi_to_f32(v.w[2 * k + 1]) * scale);
                    if (active) {
                        static_assert(W == 4, "a word of codes");
                        *(uint32_t *)(q + i * wide + half * c.cols) = code[0][i];
                    }
                }
#pragma unroll
                for (int k = 0; k < N / 2; ++k) {
                    uint32_t ta[4], tb[4];  // column j of the four: rows 0-3, rows 4-7
                    transpose4x4_bytes(code[k][0], code[k][1], code[k][2], code[k][3], ta[0], ta[1], ta[2], ta[3]);
                    transpose4x4_bytes(code[k][4], code[k][5], code[k][6], code[k][7], tb[0], tb[1], tb[2], tb[3]);
                    const int col = cg * W + 4 * k;
                    uint8_t *w = (uint8_t *)turned + (half * kGatedTile + col) * TILE_ROWS + (((rg >> 1) ^ ((col >> 3) & (PIECES - 1))) << 4) + (rg & 1) * 8;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *(uint2 *)(w + j * TILE_ROWS) = make_uint2(ta[j], tb[j]);
                }
            }
            __syncthreads();
            const int piece = t % PIECES;
#pragma unroll
            for (int i = 0; i < 2 * kGatedTile * PIECES / THREADS; ++i) {
                const int at = t / PIECES + THREADS / PIECES * i, half = at / kGatedTile, col = at % kGatedTile;
                const v4i v = __builtin_bit_cast(v4i, turned[at * PIECES + (piece ^ ((col >> 3) & (PIECES - 1)))]);
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
            for (int w = 1; w < WAVES; ++w)
                r = max(r, red[w]);
            const_cast<uint32_t *>(c.partials)[blockIdx.x] = r << 16;
        }
    }
    if constexpr (PASS == kGatedDelayed)
        quant_amax_commit<WAVES>(mx, c.amax_acc);
}

template <int PASS, bool E5M2, bool SMALL, bool GELU>
static hipError_t launch_pass(GatedGradDev &c, int64_t most, hipStream_t s)
{
    c.tiles = c.tiles_x * ((c.rows + gated_rows(PASS, SMALL) - 1) / gated_rows(PASS, SMALL));
    const unsigned n = (unsigned)std::min(c.tiles, most);
    if (PASS == kGatedAmax)
        c.n_partials = (int)n;
    hipLaunchKernelGGL((gated_grad_kernel<PASS, E5M2, SMALL, GELU>), dim3(n), dim3(gated_threads(PASS, SMALL)), 0, s, c);
    return hipGetLastError();
}

template <bool E5M2, bool GELU>
static hipError_t launch_grad(const GatedGradCall &call, GatedGradDev c, hipStream_t s)
{
    const bool small = c.tiles_x * ((c.rows + kGatedTile - 1) / kGatedTile) < 2 * (int64_t)num_cus_public();
    // each workgroup ends in a word of its own, or in an atomic: three a CU walk the tiles.  The cast has one a tile, as far as a launch goes:
    // less than 2^32 threads (2^30 rows of 128 columns are 2^23 tiles of 512).
    const int64_t few = std::min<int64_t>(3 * (int64_t)num_cus_public(), kGatedPartials), all = (int64_t)1 << 22;
    float *state = (float *)call.state;
    if (state != nullptr && !call.bootstrap) {
        c.scale = state + 17;
        c.amax_acc = (uint32_t *)state + 16;
        const hipError_t e = launch_pass<kGatedDelayed, E5M2, false, GELU>(c, few, s);
        return e == hipSuccess ? launch_delayed_update(state, false, E5M2, nullptr, 0, call.scalars, s) : e;
    }
    c.partials = call.partials;
    hipError_t e = small ? launch_pass<kGatedAmax, false, true, GELU>(c, kGatedPartials, s) : launch_pass<kGatedAmax, false, false, GELU>(c, few, s);
    if (e == hipSuccess && state != nullptr) {
        e = launch_delayed_update(state, true, E5M2, call.partials, c.n_partials, call.scalars, s);
        c.scale = state + 21;
    }
    if (e != hipSuccess)
        return e;
    return small ? launch_pass<kGatedCast, E5M2, true, GELU>(c, all, s) : launch_pass<kGatedCast, E5M2, false, GELU>(c, all, s);
}

hipError_t launch_gated_grad(const GatedGradCall &call, hipStream_t s)
{
    GatedGradDev c{};
    c.dh = (const uint16_t *)call.dh;
    c.gu = (const uint16_t *)call.gu;
    c.rows = call.M;
    c.cols = call.F;
    c.tiles_x = (call.F + kGatedTile - 1) / kGatedTile;
    c.act = gate_coef(call.gelu);
    constexpr double k = 1.5957691216057307118;  // 2 sqrt(2 / pi)
    c.slope0 = (float)k;
    c.slope1 = (float)(3 * k * 0.044715);
    c.q = call.q;
    c.qT = call.qT;
    c.scalars = call.scalars;
    if (call.gelu)
        return call.e5m2 ? launch_grad<true, true>(call, c, s) : launch_grad<false, true>(call, c, s);
    return call.e5m2 ? launch_grad<true, false>(call, c, s) : launch_grad<false, false>(call, c, s);
}

}  // namespace tweo
