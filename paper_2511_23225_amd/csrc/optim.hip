// What follows the gradients of a training step: the sum of their squares over all tensors, and the AdamW step.  gfx950 only.
#include <algorithm>
#include "kernels.h"
#include "device_utils.h"

namespace tweo {

namespace {

// ---------------------------------------------------------------------------
// The table of tensors lies in device memory; a wave finds its place in it by the running count of chunks.  A chunk is 1024
// elements of one tensor, 16 a lane; a tensor's last one may be short.
struct Entry {
    void *param;
    float *master;
    const void *grad;
    void *m, *v;
    float *m_step, *v_step;
    int64_t n;
    int64_t first_chunk;
    float weight_decay;
    uint32_t kind;  // OptimKind bits
};
static_assert(sizeof(Entry) == kOptimEntryBytes, "the size that callers are told");

constexpr int kChunk = kOptimChunk;
static_assert(kChunk == 16 * kWave, "16 elements a lane");
constexpr int kEntriesALaunch = 32;  // of the table, by value: a launch's arguments hold 4 KB

struct EntryBatch {
    Entry e[kEntriesALaunch];
};

__global__ __launch_bounds__(kWave) void optim_table_kernel(EntryBatch b, int count, Entry *table)
{
    // words, a lane each: the arguments are read and the table written once
    const uint32_t *from = (const uint32_t *)b.e;
    uint32_t *to = (uint32_t *)table;
    for (int i = threadIdx.x; i < count * (int)(sizeof(Entry) / 4); i += kWave)
        to[i] = from[i];
}

// the entry that holds chunk c
__device__ __forceinline__ int find_entry(const Entry *table, int count, int64_t c)
{
    int lo = 0, hi = count;  // table[lo].first_chunk <= c < table[hi].first_chunk
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (table[mid].first_chunk <= c)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Four consecutive elements from an address that is a multiple of four elements; with those past the tensor's end as zeros.
template <bool F32>
struct Four;
template <>
struct Four<true> {
    typedef float4 raw;
    static __device__ __forceinline__ raw load(const void *p, int64_t i) { return *(const float4 *)((const float *)p + i); }
    static __device__ __forceinline__ raw load_some(const void *p, int64_t i, int n)
    {
        const float *f = (const float *)p + i;
        return make_float4(n > 0 ? f[0] : 0.0f, n > 1 ? f[1] : 0.0f, n > 2 ? f[2] : 0.0f, n > 3 ? f[3] : 0.0f);
    }
    static __device__ __forceinline__ void widen(raw r, float (&out)[4]) { out[0] = r.x, out[1] = r.y, out[2] = r.z, out[3] = r.w; }
    static __device__ __forceinline__ void store(void *p, int64_t i, const float (&v)[4])
    {
        *(float4 *)((float *)p + i) = make_float4(v[0], v[1], v[2], v[3]);
    }
    static __device__ __forceinline__ void store_some(void *p, int64_t i, int n, const float (&v)[4])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n)
                ((float *)p)[i + k] = v[k];
    }
};
template <>
struct Four<false> {
    typedef uint2 raw;
    static __device__ __forceinline__ raw load(const void *p, int64_t i) { return *(const uint2 *)((const uint16_t *)p + i); }
    static __device__ __forceinline__ raw load_some(const void *p, int64_t i, int n)
    {
        const uint16_t *h = (const uint16_t *)p + i;
        const uint32_t e0 = n > 0 ? h[0] : 0u, e1 = n > 1 ? h[1] : 0u, e2 = n > 2 ? h[2] : 0u, e3 = n > 3 ? h[3] : 0u;
        return make_uint2(e0 | e1 << 16, e2 | e3 << 16);
    }
    static __device__ __forceinline__ void widen(raw r, float (&out)[4])
    {
        out[0] = bf16lo_to_f32(r.x), out[1] = bf16hi_to_f32(r.x), out[2] = bf16lo_to_f32(r.y), out[3] = bf16hi_to_f32(r.y);
    }
    static __device__ __forceinline__ void store(void *p, int64_t i, const float (&v)[4])
    {
        *(uint2 *)((uint16_t *)p + i) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
    static __device__ __forceinline__ void store_some(void *p, int64_t i, int n, const float (&v)[4])
    {
        const uint32_t lo = pack_bf16x2(v[0], v[1]), hi = pack_bf16x2(v[2], v[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n)
                ((uint16_t *)p)[i + k] = (uint16_t)((k < 2 ? lo : hi) >> (16 * (k & 1)));
    }
};

// ---------------------------------------------------------------------------
// Sum of squares of all gradients.  2 (bf16) or 4 bytes an element read, nothing else.  fp64 from the square on: bf16 and fp32 gradients
// have squares outside fp32's range, and a sum over 10^9 elements in fp32 would lose what a clipping threshold compares.  A wave
// takes consecutive chunks; workgroup b leaves its sum in partials[b], and one more workgroup adds those in a fixed order.
constexpr int kSumsqThreads = 256;

template <bool F32>
__device__ __forceinline__ double sumsq_chunk(const Entry &e, int64_t base)
{
    const int lane = threadIdx.x & (kWave - 1);
    typename Four<F32>::raw r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = base + 4 * (j * kWave + lane);
        const int64_t left = e.n - i;
        r[j] = left >= 4 ? Four<F32>::load(e.grad, i) : Four<F32>::load_some(e.grad, i, left > 0 ? (int)left : 0);
    }
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float g[4];
        Four<F32>::widen(r[j], g);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            s = __builtin_fma((double)g[k], (double)g[k], s);
    }
    return s;
}

__device__ __forceinline__ double workgroup_sum(double v, double *red, int threads)
{
    v = wave_reduce_sum(v);
    if ((threadIdx.x & (kWave - 1)) == 0)
        red[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < threads / kWave; ++w)
        s += red[w];
    return s;
}

__global__ __launch_bounds__(kSumsqThreads) void grad_sumsq_kernel(const Entry *__restrict__ table, int count, int64_t chunks,
                                                                   double *__restrict__ partials)
{
    const int64_t waves = (int64_t)gridDim.x * (kSumsqThreads / kWave),
                  wave = (int64_t)blockIdx.x * (kSumsqThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t from = chunks * wave / waves, to = chunks * (wave + 1) / waves;
    double s = 0.0;
    if (from < to) {
        int at = find_entry(table, count, from);
        for (int64_t c = from; c < to; ++c) {
            while (at + 1 < count && table[at + 1].first_chunk <= c)
                ++at;
            const Entry &e = table[at];
            const int64_t base = (c - e.first_chunk) * kChunk;
            s += e.kind & kOptimGradF32 ? sumsq_chunk<true>(e, base) : sumsq_chunk<false>(e, base);
        }
    }
    __shared__ double red[kSumsqThreads / kWave];
    s = workgroup_sum(s, red, kSumsqThreads);
    if (threadIdx.x == 0)
        partials[blockIdx.x] = s;
}

__global__ __launch_bounds__(kSumsqThreads) void grad_sumsq_finish_kernel(const double *__restrict__ partials, int n, double *out)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kSumsqThreads)
        s += partials[i];
    __shared__ double red[kSumsqThreads / kWave];
    s = workgroup_sum(s, red, kSumsqThreads);
    if (threadIdx.x == 0)
        *out = s;
}

// ---------------------------------------------------------------------------
// AdamW: with the clipped gradient g' = c g, c = min(1, max_norm / (sqrt(S) + 1e-6)),
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,  p = p - lr wd p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
//
// 8-bit states: a block of 256 elements shares an fp32 step for m (E4M3 codes) and one for v (E5M2: no square root is taken on the way,
// and 2^32 between the largest and the smallest).  A block is 16 lanes of a wave with 16 elements each, four at a time 64 apart, so that its
// maxima are four DPP steps and the lanes' loads lie side by side.
//
// Rounding to codes: an E4M3 or E5M2 step is 6-25 % of the value, a moment moves by 1 - b2 (0.1-5 %) a step.  Rounded to nearest, v would stay
// where it is for ever.  So the part that is cut off decides with a threshold that is spread evenly over [0, 1) along the steps t of
// one element and along the elements i of one step: u = frac(i (sqrt(2) - 1) + t (sqrt(5) - 1) / 2), as 32-bit integers: a multiplication
// and an addition, and any step can be recomputed.  Simulated over 300 steps at b2 = 0.99 (0.95, 0.999), the coded v over the exact one: mean
// 0.985 (0.983, 0.987), spread 0.25 (0.18, 0.25); with independent random numbers 0.998, 0.29 (0.23, 0.30); to nearest 1.24 (1.08, 1.14), 0.35
// (0.20, 0.36).  In bits: y, the
// scaled value times the power of two that puts the code's exponent field where fp32 has its own (codes below the normal ones
// becoming fp32's subnormals), plus the top of u below the code's last bit, shifted.
struct AdamwArgs {
    const Entry *table;
    int count;
    int64_t chunks;
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps, lr, step_size, inv_sqrt_bc2;
    double beta1_d, beta2_d, max_norm;
    uint32_t step;
    const double *grad_sumsq;
    const OptimSchedule *schedule;
};

struct StepScalars {
    float lr, step_size, inv_sqrt_bc2, clip;
    uint32_t dither;  // t times its odd factor
};

__device__ __forceinline__ float fmul(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}
__device__ __forceinline__ float fadd(float a, float b)
{
#pragma clang fp contract(off)
    return a + b;
}

// b1 m + (1 - b1) g in separate roundings: the codes of a step follow from its inputs by IEEE operations in this order alone
__device__ __forceinline__ float blend(float beta, float old, float one_minus_beta, float now)
{
    return fadd(fmul(beta, old), fmul(one_minus_beta, now));
}

// p with the new moments; v_sqrt and v_rcp are within 1 ulp, far below what the rounding of p loses
__device__ __forceinline__ float updated(float p, float m, float v, float lr_decay, const StepScalars &k, float eps)
{
    const float denom = __builtin_fmaf(__builtin_amdgcn_sqrtf(v), k.inv_sqrt_bc2, eps);
    const float change = __builtin_fmaf(lr_decay, p, k.step_size * (m * __builtin_amdgcn_rcpf(denom)));
    return p - change;
}

// maximum over the 16 lanes of a DPP row, in all of them
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v)
{
    auto step = [](uint32_t x, auto ctrl) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, decltype(ctrl)::value, 0xF, 0xF, false);
        return o > x ? o : x;
    };
    v = step(v, std::integral_constant<int, 0xB1>{});   // quad_perm: 1 0 3 2
    v = step(v, std::integral_constant<int, 0x4E>{});   // quad_perm: 2 3 0 1
    v = step(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
    v = step(v, std::integral_constant<int, 0x140>{});  // row_mirror
    return v;
}

struct BlockScale {
    float scale, step;
};
// of a block whose largest magnitude has this pattern; an infinity or a NaN makes the step NaN, and with it the block
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits, float top)
{
    const float amax = bits_to_f32(amax_bits), scale = scale_from_amax_range(amax, top);
    return {scale, amax_bits < 0x7F800000u ? 1.0f / scale : __builtin_nanf("")};
}

template <int CUT>
__device__ __forceinline__ uint32_t encode(float magnitude, float scale, float to_field, uint32_t largest, uint32_t u)
{
    const float y = fmul(fmul(magnitude, scale), to_field);
    const uint32_t code = (f32_to_bits(y) + (u >> (32 - CUT))) >> CUT;
    return code < largest ? code : largest;
}

constexpr uint32_t kDitherElement = 0x6A09E667u, kDitherStep = 0x9E3779B9u;  // 2^32 (sqrt(2) - 1), 2^32 (sqrt(5) - 1) / 2, odd

// KIND: kOptimParamF32, kOptimMaster, kOptimGradF32.  FULL: the chunk has all of its elements.
template <bool EIGHT, uint32_t KIND, bool FULL>
__device__ __forceinline__ void adamw_chunk(const Entry &e, int64_t base, const AdamwArgs &a, const StepScalars &k)
{
    constexpr bool P32 = (KIND & kOptimParamF32) != 0, MASTER = (KIND & kOptimMaster) != 0, G32 = (KIND & kOptimGradF32) != 0;
    typedef Four<P32 || MASTER> P;
    typedef Four<G32> G;
    const int lane = threadIdx.x & (kWave - 1);
    void *weights = MASTER ? (void *)e.master : e.param;
    const int64_t n = e.n;
    // the lane's four elements of pass j
    auto at = [&](int j) { return base + (EIGHT ? (lane >> 4) * 256 + j * 64 + (lane & 15) * 4 : j * 256 + lane * 4); };
    auto some = [&](int64_t i) { return n - i < 4 ? (n - i > 0 ? (int)(n - i) : 0) : 4; };
    auto load = [&](auto four, const void *p, int64_t i) {
        typedef decltype(four) F;
        return FULL || some(i) == 4 ? F::load(p, i) : F::load_some(p, i, some(i));
    };
    auto store = [&](auto four, void *p, int64_t i, const float (&x)[4]) {
        typedef decltype(four) F;
        if (FULL || some(i) == 4)
            F::store(p, i, x);
        else
            F::store_some(p, i, some(i), x);
    };
    auto load_codes = [&](const void *p, int64_t i) {
        if (FULL || some(i) == 4)
            return *(const uint32_t *)((const uint8_t *)p + i);
        uint32_t c = 0;
        for (int b = 0; b < some(i); ++b)
            c |= (uint32_t)((const uint8_t *)p)[i + b] << (8 * b);
        return c;
    };
    auto store_codes = [&](void *p, int64_t i, uint32_t c) {
        if (FULL || some(i) == 4) {
            *(uint32_t *)((uint8_t *)p + i) = c;
            return;
        }
        for (int b = 0; b < some(i); ++b)
            ((uint8_t *)p)[i + b] = (uint8_t)(c >> (8 * b));
    };
    typename P::raw pr[4];
    typename G::raw gr[4];
    float4 mr[4], vr[4];
    uint32_t mc[4], vc[4];
    float m_step = 0.0f, v_step = 0.0f;
    const int64_t block = base / 256 + (lane >> 4);
    const bool has_block = FULL || base + (lane >> 4) * 256 < n;
    if constexpr (EIGHT) {
        if (has_block) {
            m_step = e.m_step[block];
            v_step = e.v_step[block];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = at(j);
        gr[j] = load(G{}, e.grad, i);
        if constexpr (EIGHT) {
            mc[j] = load_codes(e.m, i);
            vc[j] = load_codes(e.v, i);
        } else {
            mr[j] = load(Four<true>{}, e.m, i);
            vr[j] = load(Four<true>{}, e.v, i);
        }
        pr[j] = load(P{}, weights, i);
    }
    const float lr_decay = k.lr * e.weight_decay;
    float m[4][4], v[4][4];
    uint32_t m_max = 0, v_max = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float g[4], p[4];
        G::widen(gr[j], g);
        P::widen(pr[j], p);
        if constexpr (EIGHT) {
            const v2f m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[j], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[j], true);
            const v2f v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vc[j], false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vc[j], true);
            m[j][0] = fmul(m0[0], m_step), m[j][1] = fmul(m0[1], m_step), m[j][2] = fmul(m1[0], m_step), m[j][3] = fmul(m1[1], m_step);
            v[j][0] = fmul(v0[0], v_step), v[j][1] = fmul(v0[1], v_step), v[j][2] = fmul(v1[0], v_step), v[j][3] = fmul(v1[1], v_step);
        } else {
            Four<true>::widen(mr[j], m[j]);
            Four<true>::widen(vr[j], v[j]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float gc = fmul(g[q], k.clip);
            m[j][q] = blend(a.beta1, m[j][q], a.one_minus_beta1, gc);
            v[j][q] = blend(a.beta2, v[j][q], a.one_minus_beta2, fmul(gc, gc));
            p[q] = updated(p[q], m[j][q], v[j][q], lr_decay, k, a.eps);
            if constexpr (EIGHT) {
                // what lies behind the tensor's end is zero in all of them and no maximum
                const uint32_t mb = f32_to_bits(m[j][q]) & 0x7FFFFFFFu, vb = f32_to_bits(v[j][q]) & 0x7FFFFFFFu;
                m_max = mb > m_max ? mb : m_max;
                v_max = vb > v_max ? vb : v_max;
            }
        }
        const int64_t i = at(j);
        store(P{}, weights, i, p);
        if constexpr (MASTER)
            store(Four<false>{}, e.param, i, p);
        if constexpr (!EIGHT) {
            store(Four<true>{}, e.m, i, m[j]);
            store(Four<true>{}, e.v, i, v[j]);
        }
    }
    if constexpr (EIGHT) {
        const BlockScale ms = block_scale(row_max_u32(m_max), 448.0f), vs = block_scale(row_max_u32(v_max), 57344.0f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t i = at(j);
            uint32_t mo = 0, vo = 0, u = (uint32_t)i * kDitherElement + k.dither;
#pragma unroll
            for (int q = 0; q < 4; ++q, u += kDitherElement) {
                uint32_t c = encode<20>(__builtin_fabsf(m[j][q]), ms.scale, 0x1p-120f, 0x7Eu, u);
                mo |= (c | (f32_to_bits(m[j][q]) >> 24 & 0x80u)) << (8 * q);
                c = encode<21>(__builtin_fabsf(v[j][q]), vs.scale, 0x1p-112f, 0x7Bu, u);
                // a positive second moment stays positive: it is a divisor
                vo |= (c == 0u && v[j][q] > 0.0f ? 1u : c) << (8 * q);
            }
            store_codes(e.m, i, mo);
            store_codes(e.v, i, vo);
        }
        if ((lane & 15) == 0 && has_block) {
            e.m_step[block] = ms.step;
            e.v_step[block] = vs.step;
        }
    }
}

template <bool EIGHT, bool FULL>
__device__ __forceinline__ void adamw_any(const Entry &e, int64_t base, const AdamwArgs &a, const StepScalars &k)
{
    switch (e.kind) {
    case 0: adamw_chunk<EIGHT, 0, FULL>(e, base, a, k); break;
    case kOptimGradF32: adamw_chunk<EIGHT, kOptimGradF32, FULL>(e, base, a, k); break;
    case kOptimParamF32: adamw_chunk<EIGHT, kOptimParamF32, FULL>(e, base, a, k); break;
    case kOptimParamF32 | kOptimGradF32: adamw_chunk<EIGHT, kOptimParamF32 | kOptimGradF32, FULL>(e, base, a, k); break;
    case kOptimMaster: adamw_chunk<EIGHT, kOptimMaster, FULL>(e, base, a, k); break;
    default: adamw_chunk<EIGHT, kOptimMaster | kOptimGradF32, FULL>(e, base, a, k); break;
    }
}

constexpr int kAdamwThreads = 256;

template <bool EIGHT>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(AdamwArgs a)
{
    StepScalars k{a.lr, a.step_size, a.inv_sqrt_bc2, 1.0f, a.step * kDitherStep};
    if (a.schedule != nullptr) {
        const AdamwScalars s = adamw_scalars((double)a.schedule->lr, a.beta1_d, a.beta2_d, a.schedule->step);
        k = {a.schedule->lr, s.step_size, s.inv_sqrt_bc2, 1.0f, a.schedule->step * kDitherStep};
    }
    if (a.grad_sumsq != nullptr) {
        const double norm = __builtin_sqrt(*a.grad_sumsq);
        if (!(norm < __builtin_inf()))
            return;  // a gradient that is not finite: no tensor changes
        const double c = a.max_norm / (norm + 1e-6);
        k.clip = c < 1.0 ? (float)c : 1.0f;
    }
    const int64_t waves = (int64_t)gridDim.x * (kAdamwThreads / kWave),
                  wave = (int64_t)blockIdx.x * (kAdamwThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t from = a.chunks * wave / waves, to = a.chunks * (wave + 1) / waves;
    if (from >= to)
        return;
    int at = find_entry(a.table, a.count, from);
    for (int64_t c = from; c < to; ++c) {
        while (at + 1 < a.count && a.table[at + 1].first_chunk <= c)
            ++at;
        const Entry &e = a.table[at];
        const int64_t base = (c - e.first_chunk) * kChunk;
        if (base + kChunk <= e.n)
            adamw_any<EIGHT, true>(e, base, a, k);
        else
            adamw_any<EIGHT, false>(e, base, a, k);
    }
}

constexpr int kCus = 256;

}  // namespace

int64_t optim_chunks(int64_t n) { return (n + kChunk - 1) / kChunk; }

hipError_t launch_optim_table(const OptimTensor *tensors, int count, void *table, hipStream_t s)
{
    int64_t chunk = 0;
    for (int from = 0; from < count; from += kEntriesALaunch) {
        EntryBatch b{};
        const int some = std::min(kEntriesALaunch, count - from);
        for (int i = 0; i < some; ++i) {
            const OptimTensor &t = tensors[from + i];
            b.e[i] = {t.param, t.master, t.grad, t.m, t.v, t.m_step, t.v_step, t.n, chunk, t.weight_decay, t.kind};
            chunk += optim_chunks(t.n);
        }
        hipLaunchKernelGGL(optim_table_kernel, dim3(1), dim3(kWave), 0, s, b, some, (Entry *)table + from);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

hipError_t launch_grad_sumsq(const void *table, int count, int64_t chunks, double *out, double *partials, hipStream_t s)
{
    const int groups = (int)std::min<int64_t>((chunks + 3) / 4, kSumsqPartials);
    hipLaunchKernelGGL(grad_sumsq_kernel, dim3(groups), dim3(kSumsqThreads), 0, s, (const Entry *)table, count, chunks, partials);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(grad_sumsq_finish_kernel, dim3(1), dim3(kSumsqThreads), 0, s, partials, groups, out);
    return hipGetLastError();
}

hipError_t launch_adamw(const void *table, int count, int64_t chunks, bool eight_bits, const AdamwCall &c, hipStream_t s)
{
    const AdamwScalars k = adamw_scalars(c.lr, c.beta1, c.beta2, c.step);
    const AdamwArgs a{(const Entry *)table, count, chunks, (float)c.beta1, (float)(1.0 - c.beta1), (float)c.beta2, (float)(1.0 - c.beta2),
                      (float)c.eps, (float)c.lr, k.step_size, k.inv_sqrt_bc2, c.beta1, c.beta2, c.max_norm, c.step, c.grad_sumsq, c.schedule};
    const unsigned groups = (unsigned)std::min<int64_t>((chunks + 3) / 4, 4 * kCus);
    if (eight_bits)
        hipLaunchKernelGGL(adamw_kernel<true>, dim3(groups), dim3(kAdamwThreads), 0, s, a);
    else
        hipLaunchKernelGGL(adamw_kernel<false>, dim3(groups), dim3(kAdamwThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace tweo
