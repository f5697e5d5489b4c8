// What follows the gradients of a training step: the sum of their squares over all tensors, and the AdamW step.  gfx950 only.
// Times in the comments: a call among others in a replayed graph, on three sets of tensors in turn.
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

// The table's addresses are of global memory, the table itself is read through the scalar cache: told to the compiler, which takes what it
// reads from memory for an address in any space (FLAT accesses) and the table for something that the stores could change.
#define GLOBAL __attribute__((address_space(1)))
#define CONSTANT __attribute__((address_space(4)))
typedef const CONSTANT Entry *Table;

// The entry that holds chunk c: the wave's lanes look at 64 entries at once, so that up to 64 tensors take one load's time and
// up to 4096 two.  (Halving took six to eight loads that wait for each other.)
__device__ __forceinline__ int find_entry(Table table, int count, int64_t c)
{
    const int lane = threadIdx.x & (kWave - 1);
    int from = 0, to = count;  // table[from].first_chunk <= c
    while (to - from > 1) {
        const int step = (to - from + kWave - 1) / kWave, i = from + lane * step;
        const bool below = i < to && table[i].first_chunk <= c;
        const int last = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below)) - 1;  // lane 0's is always below
        from += last * step;
        to = from + step < to ? from + step : to;
    }
    return __builtin_amdgcn_readfirstlane(from);
}

// Loads and stores of four consecutive elements, `at` bytes behind a base that all lanes share.  ONCE: past the caches, for a model whose
// buffers together are more than the memory-side cache keeps from one step to the next.
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <bool F32>
struct Four;
template <>
struct Four<true> {
    typedef f32x4 raw;
    static constexpr uint32_t kBytes = 4;
    template <bool ONCE>
    static __device__ __forceinline__ raw load(const GLOBAL uint8_t *p, uint32_t at)
    {
        const GLOBAL raw *q = (const GLOBAL raw *)(p + at);
        return ONCE ? __builtin_nontemporal_load(q) : *q;
    }
    static __device__ __forceinline__ raw load_some(const GLOBAL uint8_t *p, uint32_t at, int n)
    {
        const GLOBAL float *f = (const GLOBAL float *)(p + at);
        return raw{n > 0 ? f[0] : 0.0f, n > 1 ? f[1] : 0.0f, n > 2 ? f[2] : 0.0f, n > 3 ? f[3] : 0.0f};
    }
    static __device__ __forceinline__ void widen(raw r, float (&out)[4]) { out[0] = r[0], out[1] = r[1], out[2] = r[2], out[3] = r[3]; }
    template <bool ONCE>
    static __device__ __forceinline__ void store(GLOBAL uint8_t *p, uint32_t at, const float (&v)[4])
    {
        GLOBAL raw *q = (GLOBAL raw *)(p + at);
        const raw r{v[0], v[1], v[2], v[3]};
        if constexpr (ONCE)
            __builtin_nontemporal_store(r, q);
        else
            *q = r;
    }
    static __device__ __forceinline__ void store_some(GLOBAL uint8_t *p, uint32_t at, int n, const float (&v)[4])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n)
                ((GLOBAL float *)(p + at))[k] = v[k];
    }
};
// (half the bytes of a line at a time: measured slower past the caches)
template <>
struct Four<false> {
    typedef uint32_t raw __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kBytes = 2;
    template <bool>
    static __device__ __forceinline__ raw load(const GLOBAL uint8_t *p, uint32_t at) { return *(const GLOBAL raw *)(p + at); }
    static __device__ __forceinline__ raw load_some(const GLOBAL uint8_t *p, uint32_t at, int n)
    {
        const GLOBAL uint16_t *h = (const GLOBAL uint16_t *)(p + at);
        const uint32_t e0 = n > 0 ? h[0] : 0u, e1 = n > 1 ? h[1] : 0u, e2 = n > 2 ? h[2] : 0u, e3 = n > 3 ? h[3] : 0u;
        return raw{e0 | e1 << 16, e2 | e3 << 16};
    }
    static __device__ __forceinline__ void widen(raw r, float (&out)[4])
    {
        out[0] = bf16lo_to_f32(r.x), out[1] = bf16hi_to_f32(r.x), out[2] = bf16lo_to_f32(r.y), out[3] = bf16hi_to_f32(r.y);
    }
    template <bool>
    static __device__ __forceinline__ void store(GLOBAL uint8_t *p, uint32_t at, const float (&v)[4])
    {
        *(GLOBAL raw *)(p + at) = raw{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
    static __device__ __forceinline__ void store_some(GLOBAL uint8_t *p, uint32_t at, int n, const float (&v)[4])
    {
        const uint32_t lo = pack_bf16x2(v[0], v[1]), hi = pack_bf16x2(v[2], v[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n)
                ((GLOBAL uint16_t *)(p + at))[k] = (uint16_t)((k < 2 ? lo : hi) >> (16 * (k & 1)));
    }
};
// four codes
struct Codes {
    typedef uint32_t raw;
    static constexpr uint32_t kBytes = 1;
    template <bool>
    static __device__ __forceinline__ raw load(const GLOBAL uint8_t *p, uint32_t at) { return *(const GLOBAL uint32_t *)(p + at); }
    static __device__ __forceinline__ raw load_some(const GLOBAL uint8_t *p, uint32_t at, int n)
    {
        const GLOBAL uint8_t *c = p + at;
        const uint32_t c0 = n > 0 ? c[0] : 0u, c1 = n > 1 ? c[1] : 0u, c2 = n > 2 ? c[2] : 0u, c3 = n > 3 ? c[3] : 0u;
        return c0 | c1 << 8 | c2 << 16 | c3 << 24;
    }
    template <bool>
    static __device__ __forceinline__ void store(GLOBAL uint8_t *p, uint32_t at, raw c) { *(GLOBAL uint32_t *)(p + at) = c; }
    static __device__ __forceinline__ void store_some(GLOBAL uint8_t *p, uint32_t at, int n, raw c)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n)
                (p + at)[k] = (uint8_t)(c >> (8 * k));
    }
};
// a buffer's element `base`, the same for all lanes
template <typename F>
__device__ __forceinline__ GLOBAL uint8_t *from(const void *p, int64_t base)
{
    return (GLOBAL uint8_t *)p + base * F::kBytes;
}
template <typename F, bool FULL, bool ONCE>
__device__ __forceinline__ typename F::raw load4(const GLOBAL uint8_t *p, uint32_t element, int left)
{
    if (FULL || left >= 4)
        return F::template load<ONCE>(p, element * F::kBytes);
    return F::load_some(p, element * F::kBytes, left);
}
template <typename F, bool FULL, bool ONCE, typename V>
__device__ __forceinline__ void store4(GLOBAL uint8_t *p, uint32_t element, int left, const V &v)
{
    if (FULL || left >= 4)
        F::template store<ONCE>(p, element * F::kBytes, v);
    else
        F::store_some(p, element * F::kBytes, left, v);
}

// ---------------------------------------------------------------------------
// Sum of squares of all gradients.  2 (bf16) or 4 bytes an element read, nothing else.  fp64 from the square on: bf16 and fp32 gradients
// have squares outside fp32's range, and a sum over 10^9 elements in fp32 would lose what a clipping threshold compares.  A wave
// takes consecutive chunks, four (fp32: two) at a time where the tensor has them: 8 KB under way in each.  Workgroup b leaves its sum in
// partials[b], and one more workgroup adds those in a fixed order: a counter at which the last one is found takes 12 ns a workgroup.
// 205 M bf16 gradients 68 us, 6.0 TB/s, what tweo_amax reads at; a chunk of 8-byte loads at a time 83; 3 M in 61 tensors 7.5, two launches.
constexpr int kSumsqThreads = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// whole chunks: 16 bytes a lane and load, all of them under way at once
template <bool F32, bool ONCE, int CHUNKS>
__device__ __forceinline__ double sumsq_whole(const GLOBAL uint8_t *grad)
{
    constexpr int LOADS = CHUNKS * kChunk * (F32 ? 4 : 2) / (16 * kWave);
    const GLOBAL u32x4 *p = (const GLOBAL u32x4 *)grad + (threadIdx.x & (kWave - 1));
    u32x4 r[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
        r[j] = ONCE ? __builtin_nontemporal_load(p + j * kWave) : p[j * kWave];
    double s[2] = {0.0, 0.0};
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (F32) {
                const double g = (double)bits_to_f32(r[j][k]);
                s[k & 1] = __builtin_fma(g, g, s[k & 1]);
            } else {
                const double lo = (double)bf16lo_to_f32(r[j][k]), hi = (double)bf16hi_to_f32(r[j][k]);
                s[0] = __builtin_fma(lo, lo, s[0]);
                s[1] = __builtin_fma(hi, hi, s[1]);
            }
        }
    return s[0] + s[1];
}

// the last chunk of a tensor
template <bool F32>
__device__ __forceinline__ double sumsq_rest(const GLOBAL uint8_t *grad, int n)
{
    const uint32_t first = 4 * (threadIdx.x & (kWave - 1));
    typename Four<F32>::raw r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        r[j] = load4<Four<F32>, false, false>(grad, first + 256 * j, n - (int)first - 256 * j);
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

// chunks c to `to` of one tensor (no further than its end); how many of them were taken
template <bool F32, bool ONCE>
__device__ __forceinline__ int sumsq_step(const CONSTANT Entry &e, int64_t c, int64_t to, double &s)
{
    const int64_t base = (c - e.first_chunk) * kChunk, n = e.n - base;
    const GLOBAL uint8_t *grad = from<Four<F32>>(e.grad, base);
    constexpr int MANY = F32 ? 2 : 4;
    if (n >= MANY * kChunk && to - c >= MANY) {
        s += sumsq_whole<F32, ONCE, MANY>(grad);
        return MANY;
    }
    s += n >= kChunk ? sumsq_whole<F32, ONCE, 1>(grad) : sumsq_rest<F32>(grad, (int)n);
    return 1;
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

template <bool ONCE>
__global__ __launch_bounds__(kSumsqThreads) void grad_sumsq_kernel(const Entry *entries, int count, int64_t chunks,
                                                                   double *__restrict__ partials)
{
    const int64_t waves = (int64_t)gridDim.x * (kSumsqThreads / kWave),
                  wave = (int64_t)blockIdx.x * (kSumsqThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t from = chunks * wave / waves, to = chunks * (wave + 1) / waves;
    const Table table = (Table)entries;
    double s = 0.0;
    for (int64_t c = from; c < to;) {
        const CONSTANT Entry &e = table[find_entry(table, count, c)];
        const int64_t end = e.first_chunk + (e.n + kChunk - 1) / kChunk, stop = end < to ? end : to;
        while (c < stop)
            c += e.kind & kOptimGradF32 ? sumsq_step<true, ONCE>(e, c, stop, s) : sumsq_step<false, ONCE>(e, c, stop, s);
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
// Bound by memory: 28 B an element with fp32 states beside an fp32 copy, 22 without; 16 and 10 with 8-bit states.  A wave takes
// one chunk, all of whose loads (16, with 8-bit states 18, of 4 to 16 bytes a lane) are under way before the first is waited for, and
// workgroups walk the tensors in order: 51 M elements with master, fp32 states 241 us (6.0 TB/s), 205 M with 8-bit states 580 (5.7), without
// master 374 (5.5, half of its time the SIMDs issue).  Persistent waves, each on a run of chunks of its own, took 301, 703 and
// 450; persistent ones in turns, the streams of all side by side, 284 and 665.
//
// 8-bit states: a block of 256 elements shares an fp32 step for m (E4M3 codes) and one for v (E5M2: no square root is taken on the way,
// and 2^32 between the largest and the smallest).  A block is 16 lanes of a wave with 16 elements each, four at a time 64 apart, so that its
// maxima are four DPP steps and the lanes' loads lie side by side.
//
// Rounding to codes: an E4M3 or E5M2 step is 6-25 % of the value, a moment moves by 1 - b2 (0.1-5 %) a step.  Rounded to nearest,
// v would stay where it is for ever.  So the part that is cut off decides with a threshold that is spread evenly over [0, 1)
// along the steps t of one element and along the elements i of one step: u = frac(i (sqrt(2) - 1) + t (sqrt(5) - 1) / 2), as
// 32-bit integers: a multiplication and an addition, and any step can be recomputed.  Simulated over 300 steps at b2 = 0.99
// (0.95, 0.999), the coded v over the exact one: mean 0.985 (0.983, 0.987), spread 0.25 (0.18, 0.25); with independent random
// numbers 0.998, 0.29 (0.23, 0.30); to nearest 1.24 (1.08, 1.14), 0.35 (0.20, 0.36).  In bits: y, the scaled value times the
// power of two that puts the code's exponent field where fp32 has its own (codes below the normal ones becoming fp32's
// subnormals), plus the top of u below the code's last bit, shifted.
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

// A finite gradient whose square has no place in fp32 counts as 2^63 or -2^63, in both moments: an infinite v would keep its parameter
// where it is for ever, and in 8 bits its block would be NaN from the next step on.  Infinities and NaN stay.  (Looked for in four
// gradients at a time: 205 M elements with 8-bit states 573.5 us, now 574.0, without master 378 and 382.)
__device__ __forceinline__ void hold_square(float (&g)[4])
{
    constexpr float kMost = 0x1p63f;
    const float most = __builtin_fmaxf(__builtin_fmaxf(__builtin_fabsf(g[0]), __builtin_fabsf(g[1])),
                                       __builtin_fmaxf(__builtin_fabsf(g[2]), __builtin_fabsf(g[3])));  // (of those that are no NaN)
    if (__builtin_expect(most > kMost, 0)) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (__builtin_fabsf(g[q]) > kMost && __builtin_fabsf(g[q]) < __builtin_inff())
                g[q] = __builtin_copysignf(kMost, g[q]);
    }
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

// least: 1 for what must not become zero
template <int CUT>
__device__ __forceinline__ uint32_t encode(float magnitude, float scale, float to_field, uint32_t least, uint32_t largest, uint32_t u)
{
    const float y = fmul(fmul(magnitude, scale), to_field);
    const uint32_t code = (f32_to_bits(y) + (u >> (32 - CUT))) >> CUT;
    const uint32_t up = code > least ? code : least;
    return up < largest ? up : largest;
}

constexpr uint32_t kDitherElement = 0x6A09E667u, kDitherStep = 0x9E3779B9u;  // 2^32 (sqrt(2) - 1), 2^32 (sqrt(5) - 1) / 2, odd

// What a step needs beside its tensors; false: nothing may change.  With a schedule every wave takes the powers, quotients and the root
// for itself, while its loads are under way: 51 M elements with fp32 states 241 us, with a schedule 248; 3 M in 61 tensors with 8-bit
// ones 15.5 and 16.8; 205 M 575 and 555.
__device__ __forceinline__ bool step_scalars(const AdamwArgs &a, StepScalars &k)
{
    k = {a.lr, a.step_size, a.inv_sqrt_bc2, 1.0f, a.step * kDitherStep};
    if (a.schedule != nullptr) {
        const AdamwScalars s = adamw_scalars((double)a.schedule->lr, a.beta1_d, a.beta2_d, a.schedule->step);
        k = {a.schedule->lr, s.step_size, s.inv_sqrt_bc2, 1.0f, a.schedule->step * kDitherStep};
    }
    if (a.grad_sumsq != nullptr) {
        const double norm = __builtin_sqrt(*a.grad_sumsq);
        if (!(norm < __builtin_inf()))
            return false;  // a gradient that is not finite
        const double c = a.max_norm / (norm + 1e-6);
        k.clip = c < 1.0 ? (float)c : 1.0f;
    }
    return true;
}

// KIND: kOptimParamF32, kOptimMaster, kOptimGradF32.  FULL: the chunk has all of its elements.  ONCE: see Four.
template <bool EIGHT, bool ONCE, uint32_t KIND, bool FULL>
__device__ __forceinline__ void adamw_chunk(const CONSTANT Entry &e, int64_t base, const AdamwArgs &a)
{
    constexpr bool P32 = (KIND & kOptimParamF32) != 0, MASTER = (KIND & kOptimMaster) != 0, G32 = (KIND & kOptimGradF32) != 0;
    typedef Four<P32 || MASTER> P;
    typedef Four<G32> G;
    typedef std::conditional_t<EIGHT, Codes, Four<true>> S;
    // with an fp32 copy nothing but the optimizer reads it; a parameter by itself is what the next forward pass reads
    constexpr bool P_ONCE = ONCE && MASTER;
    const int lane = threadIdx.x & (kWave - 1);
    GLOBAL uint8_t *const weights = from<P>(MASTER ? (void *)e.master : e.param, base), *const param = from<Four<false>>(e.param, base),
                          *const em = from<S>(e.m, base), *const ev = from<S>(e.v, base);
    const GLOBAL uint8_t *const grad = from<G>(e.grad, base);
    const int n = FULL ? kChunk : (int)(e.n - base);  // of the chunk
    // the lane's four elements of pass j begin at `first` + j * STEP
    constexpr int STEP = EIGHT ? 64 : 256;
    const uint32_t first = EIGHT ? (lane >> 4) * 256 + (lane & 15) * 4 : lane * 4;
    const int left = n - (int)first;
    typename P::raw pr[4];
    typename G::raw gr[4];
    typename S::raw mr[4], vr[4];
    float m_step = 0.0f, v_step = 0.0f;
    const int64_t block = base / 256 + (lane >> 4);
    const bool has_block = FULL || (lane >> 4) * 256 < n;
    if constexpr (EIGHT) {
        if (has_block) {
            m_step = ((const GLOBAL float *)e.m_step)[block];
            v_step = ((const GLOBAL float *)e.v_step)[block];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t i = first + j * STEP;
        gr[j] = load4<G, FULL, ONCE>(grad, i, left - j * STEP);
        mr[j] = load4<S, FULL, ONCE>(em, i, left - j * STEP);
        vr[j] = load4<S, FULL, ONCE>(ev, i, left - j * STEP);
        pr[j] = load4<P, FULL, P_ONCE>(weights, i, left - j * STEP);
    }
    // while these are on their way
    StepScalars k;
    if (!step_scalars(a, k))
        return;
    const float lr_decay = k.lr * e.weight_decay;
    float m[4][4], v[4][4];
    uint32_t m_max = 0, v_max = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float g[4], p[4];
        G::widen(gr[j], g);
        P::widen(pr[j], p);
        if constexpr (EIGHT) {
            const v2f m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mr[j], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mr[j], true);
            const v2f v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vr[j], false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vr[j], true);
            m[j][0] = fmul(m0[0], m_step), m[j][1] = fmul(m0[1], m_step), m[j][2] = fmul(m1[0], m_step), m[j][3] = fmul(m1[1], m_step);
            v[j][0] = fmul(v0[0], v_step), v[j][1] = fmul(v0[1], v_step), v[j][2] = fmul(v1[0], v_step), v[j][3] = fmul(v1[1], v_step);
        } else {
            S::widen(mr[j], m[j]);
            S::widen(vr[j], v[j]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            g[q] = fmul(g[q], k.clip);
        hold_square(g);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float gc = g[q];
            m[j][q] = blend(a.beta1, m[j][q], a.one_minus_beta1, gc);
            v[j][q] = blend(a.beta2, v[j][q], a.one_minus_beta2, fmul(gc, gc));
            p[q] = updated(p[q], m[j][q], v[j][q], lr_decay, k, a.eps);
            if constexpr (EIGHT) {
                // as patterns a NaN is the largest, whatever its sign in v; what lies behind the tensor's end is zero and no maximum
                const uint32_t mb = f32_to_bits(m[j][q]) & 0x7FFFFFFFu, vb = f32_to_bits(v[j][q]);
                m_max = mb > m_max ? mb : m_max;
                v_max = vb > v_max ? vb : v_max;
            }
        }
        const uint32_t i = first + j * STEP;
        store4<P, FULL, P_ONCE>(weights, i, left - j * STEP, p);
        if constexpr (MASTER)
            store4<Four<false>, FULL, false>(param, i, left - j * STEP, p);
        if constexpr (!EIGHT) {
            store4<S, FULL, ONCE>(em, i, left - j * STEP, m[j]);
            store4<S, FULL, ONCE>(ev, i, left - j * STEP, v[j]);
        }
    }
    if constexpr (EIGHT) {
        const BlockScale ms = block_scale(row_max_u32(m_max), 448.0f), vs = block_scale(row_max_u32(v_max), 57344.0f);
        const uint32_t u0 = ((uint32_t)base + first) * kDitherElement + k.dither;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t mo = 0, vo = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t u = u0 + (uint32_t)(j * STEP + q) * kDitherElement, mb = f32_to_bits(m[j][q]), vb = f32_to_bits(v[j][q]);
                const uint32_t mc = encode<20>(__builtin_fabsf(m[j][q]), ms.scale, 0x1p-120f, 0u, 0x7Eu, u);
                mo |= (mc | (mb >> 24 & 0x80u)) << (8 * q);
                // a positive second moment stays positive: it is a divisor
                vo |= encode<21>(__builtin_fabsf(v[j][q]), vs.scale, 0x1p-112f, vb < 1u ? vb : 1u, 0x7Bu, u) << (8 * q);
            }
            store4<S, FULL, false>(em, first + j * STEP, left - j * STEP, mo);
            store4<S, FULL, false>(ev, first + j * STEP, left - j * STEP, vo);
        }
        if ((lane & 15) == 0 && has_block) {
            ((GLOBAL float *)e.m_step)[block] = ms.step;
            ((GLOBAL float *)e.v_step)[block] = vs.step;
        }
    }
}

template <bool EIGHT, bool ONCE, bool FULL>
__device__ __forceinline__ void adamw_any(const CONSTANT Entry &e, int64_t base, const AdamwArgs &a)
{
    switch (e.kind) {
    case 0: adamw_chunk<EIGHT, ONCE, 0, FULL>(e, base, a); break;
    case kOptimGradF32: adamw_chunk<EIGHT, ONCE, kOptimGradF32, FULL>(e, base, a); break;
    case kOptimParamF32: adamw_chunk<EIGHT, ONCE, kOptimParamF32, FULL>(e, base, a); break;
    case kOptimParamF32 | kOptimGradF32: adamw_chunk<EIGHT, ONCE, kOptimParamF32 | kOptimGradF32, FULL>(e, base, a); break;
    case kOptimMaster: adamw_chunk<EIGHT, ONCE, kOptimMaster, FULL>(e, base, a); break;
    default: adamw_chunk<EIGHT, ONCE, kOptimMaster | kOptimGradF32, FULL>(e, base, a); break;
    }
}

constexpr int kAdamwThreads = 256;

template <bool EIGHT, bool ONCE>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(AdamwArgs a)
{
    const int64_t waves = (int64_t)gridDim.x * (kAdamwThreads / kWave),
                  wave = (int64_t)blockIdx.x * (kAdamwThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Table table = (Table)a.table;
    for (int64_t c = wave; c < a.chunks; c += waves) {
        const CONSTANT Entry &e = table[find_entry(table, a.count, c)];
        const int64_t base = (c - e.first_chunk) * kChunk;
        if (base + kChunk <= e.n)
            adamw_any<EIGHT, ONCE, true>(e, base, a);
        else
            adamw_any<EIGHT, ONCE, false>(e, base, a);
    }
}

constexpr int64_t kAdamwMostGroups = 1 << 20;

// Whether buffers of so many bytes an element are more than the memory-side cache (256 MB) gives back to the next step.  One step after the
// other, without and with accesses past the caches: fp32 states beside a master, 28 B an element, 3 M elements 15.3 us and 17.7, 5 M 24.7 and
// 25.9, 7 M 36.9 and 34.8, 20 M 108 and 87; 8-bit ones, 16 B, 5 M 19.0 and 20.7, 10 M 32.8 and 30.9, 20 M 67 and 58.
// (The norm, bf16 gradients: 103 MB 22.9 and 22.9, 411 MB 77 and 68.)  The callers count what was measured here, 28, 16 and 2 bytes an
// element, whatever a table holds: without a master (22 and 10) it is from 124 and 98 MB on, of fp32 gradients from 315 MB on (200 MB
// 40 us, 5.0 TB/s; 280 MB 53.5; 320 MB 52.8, 6.1 TB/s).
constexpr int64_t kKeptBytes = 150 << 20;
bool past_caches(int64_t chunks, int64_t bytes) { return chunks * kChunk * bytes > kKeptBytes; }

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
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(kSumsqThreads), 0, s, (const Entry *)table, count, chunks, partials); };
    past_caches(chunks, 2) ? go(grad_sumsq_kernel<true>) : go(grad_sumsq_kernel<false>);
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
    const unsigned groups = (unsigned)std::min<int64_t>((chunks + 3) / 4, kAdamwMostGroups);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(kAdamwThreads), 0, s, a); };
    if (past_caches(chunks, eight_bits ? 16 : 28))
        eight_bits ? go(adamw_kernel<true, true>) : go(adamw_kernel<false, true>);
    else
        eight_bits ? go(adamw_kernel<true, false>) : go(adamw_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace tweo
