// Heads of queries and keys (gfx950): rotation by position, norm of each head with the rotation behind it, and the norm's gradients.
//
//   angle  = position * freq (fp64), taken modulo a turn before it becomes fp32
//   R      : (a, b) -> scale * (a cos - b sin, b cos + a sin) on the pairs of the first `rot` values of a head, the others as they are
//   rotary : y = R x, or (transposed, the gradient) R^T x
//   norm   : xhat = x * rstd, rstd = 1 / sqrt(mean(x^2) + eps), y = R (xhat * gain)
//   grad   : d = R^T dy, w = d * gain, dx = rstd * (w - xhat * mean(w * xhat)), dgain = sum over tokens and heads of d * xhat
//
// A head belongs to a team of 1 to 32 lanes (a power of two, 16 values each) that hold both members of a pair in one lane: in 16-byte pieces, or, where
// width and turned part do not divide so, in words or single elements (HeadsLane).  The angles of a
// workgroup's tokens are worked out once, one a thread, into LDS and serve all heads; nothing else is shared, so
// memory bounds the large calls.
#include <algorithm>
#include "device_utils.h"
#include "kernels.h"

namespace tweo {

constexpr int kHeadsThreads = 256, kHeadsAngles = 2048, kHeadsTokens = 64;  // of a workgroup; angles (16 KB) and tokens at a time

struct HeadsSide {
    const uint16_t *x, *dy, *gain;
    uint16_t *y;
    int64_t x_token, x_head, dy_token, dy_head, y_token, y_head;
    int heads;
    // what a workgroup takes at a time: so many heads of so many tokens; `splits` workgroups share the heads of a token.  The gradients'
    // go on in steps of all workgroups' tokens.
    int block_heads, block_tokens, splits, blocks;
};
struct HeadsDev {
    HeadsSide side[2];
    int64_t tokens;
    int dim, rot;
    const int64_t *positions;
    const double *freqs;
    float scale, eps, sign;  // sign: of the angle
    float *partials;         // grad: a row of dim for each workgroup
};

// ---- where a lane's eight pairs lie: in 8 / V chunks of V pairs, chunk l + LANES k of the head's (V pairs each: of the turned part first, then
// of what is left, two by two).  a, b: the members of a pair, or of what is not turned, what lies there.
template <bool PAIRS, int V, int LANES>
struct HeadsLane {
    static constexpr int PER = 8, CHUNKS = 8 / V, WORDS = V == 1 ? 16 : 8;
    static_assert(V == 1 || V == 2 || V == 8, "elements, words or 16-byte pieces");
    typedef uint32_t vec __attribute__((ext_vector_type(V / 2 > 1 ? V / 2 : 2), aligned(2)));  // any even address will do
    typedef uint32_t word __attribute__((aligned(2)));
    int at_a[CHUNKS], at_b[CHUNKS];  // first elements, -1: none
    int turned, first;
    __device__ __forceinline__ HeadsLane(int l, int dim, int rot) : turned((rot >> 1) / V), first(l)
    {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const int c = l + LANES * k, rest = rot + 2 * V * (c - turned);
            const bool turns = c < turned;
            const int i = turns ? (PAIRS ? 2 * V * c : V * c) : rest, j = turns && !PAIRS ? (rot >> 1) + V * c : i + V;
            at_a[k] = i < dim ? i : -1;
            at_b[k] = j < dim ? j : -1;
        }
    }
    __device__ __forceinline__ bool rotates(int e) const { return first + LANES * (e / V) < turned; }
    __device__ __forceinline__ int angle(int e) const { return V * (first + LANES * (e / V)) + e % V; }
    // a column of the head, or -1
    __device__ __forceinline__ int column(int e, bool second) const
    {
        const int k = e / V, pos = PAIRS ? 2 * (e % V) + second : second ? V + e % V : e % V, from = pos < V ? at_a[k] : at_b[k];
        return from < 0 ? -1 : from + pos % V;
    }
    struct Raw {
        uint32_t w[WORDS];
    };
    template <bool ONCE>
    static __device__ __forceinline__ void fetch_chunk(const uint16_t *p, int at, uint32_t *w)
    {
        if constexpr (V == 8) {
            vec v = {0, 0, 0, 0};
            if (at >= 0)
                v = ONCE ? __builtin_nontemporal_load((const vec *)(p + at)) : *(const vec *)(p + at);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = v[k];
        } else if constexpr (V == 2) {
            *w = at >= 0 ? *(const word *)(p + at) : 0u;
        } else {
            *w = at >= 0 ? (uint32_t)p[at] : 0u;
        }
    }
    static __device__ __forceinline__ void store_chunk(uint16_t *p, int at, const uint32_t *w)
    {
        if (at < 0)
            return;
        if constexpr (V == 8)
            *(vec *)(p + at) = vec{w[0], w[1], w[2], w[3]};
        else if constexpr (V == 2)
            *(word *)(p + at) = *w;
        else
            p[at] = (uint16_t)*w;
    }
    template <bool ONCE>
    __device__ __forceinline__ Raw fetch(const uint16_t *p) const
    {
        constexpr int N = WORDS / (2 * CHUNKS);
        Raw r;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            fetch_chunk<ONCE>(p, at_a[k], r.w + 2 * N * k);
            fetch_chunk<ONCE>(p, at_b[k], r.w + 2 * N * k + N);
        }
        return r;
    }
    __device__ __forceinline__ void widen(const Raw &r, float (&a)[PER], float (&b)[PER]) const
    {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if constexpr (V == 1) {
                a[e] = bits_to_f32(r.w[2 * e] << 16);
                b[e] = bits_to_f32(r.w[2 * e + 1] << 16);
            } else if constexpr (PAIRS) {
                a[e] = bf16lo_to_f32(r.w[e]);
                b[e] = bf16hi_to_f32(r.w[e]);
            } else {
                const uint32_t wa = r.w[e / V * V + (e % V) / 2], wb = r.w[e / V * V + V / 2 + (e % V) / 2];
                a[e] = e & 1 ? bf16hi_to_f32(wa) : bf16lo_to_f32(wa);
                b[e] = e & 1 ? bf16hi_to_f32(wb) : bf16lo_to_f32(wb);
            }
        }
    }
    __device__ __forceinline__ void store(uint16_t *p, const float (&a)[PER], const float (&b)[PER]) const
    {
        constexpr int N = WORDS / (2 * CHUNKS);
        uint32_t w[WORDS];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if constexpr (V == 1) {
                const uint32_t d = pack_bf16x2(a[e], b[e]);
                w[2 * e] = d;
                w[2 * e + 1] = d >> 16;
            } else if constexpr (PAIRS) {
                w[e] = pack_bf16x2(a[e], b[e]);
            } else if (e % 2 == 0) {
                w[e / V * V + (e % V) / 2] = pack_bf16x2(a[e], a[e + 1]);
                w[e / V * V + V / 2 + (e % V) / 2] = pack_bf16x2(b[e], b[e + 1]);
            }
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            store_chunk(p, at_a[k], w + 2 * N * k);
            store_chunk(p, at_b[k], w + 2 * N * k + N);
        }
    }
};

// ---- sums over a team of LANES neighbouring lanes: exchanges within a row of 16 by DPP
template <int CTRL>
__device__ __forceinline__ float dpp_add_f32(float v)
{
    const int o = __builtin_amdgcn_update_dpp((int)f32_to_bits(v), (int)f32_to_bits(v), CTRL, 0xF, 0xF, false);
    return v + bits_to_f32((uint32_t)o);
}
// v of this lane and of lane ^ OFF, 16 or 32, without the LDS (through which sixteen sums over three steps took 1 of 8 us)
template <int OFF>
__device__ __forceinline__ float add_across(float v)
{
    typedef uint32_t pair __attribute__((ext_vector_type(2)));
    const uint32_t b = f32_to_bits(v);
    const pair r = OFF == 16 ? __builtin_bit_cast(pair, __builtin_amdgcn_permlane16_swap(b, b, false, false))
                             : __builtin_bit_cast(pair, __builtin_amdgcn_permlane32_swap(b, b, false, false));
    return bits_to_f32(r[0]) + bits_to_f32(r[1]);
}
template <int LANES>
__device__ __forceinline__ float team_sum(float v)
{
    if constexpr (LANES >= 2)
        v = dpp_add_f32<0xB1>(v);  // lane ^ 1
    if constexpr (LANES >= 4)
        v = dpp_add_f32<0x4E>(v);  // lane ^ 2
    if constexpr (LANES >= 8)
        v = dpp_add_f32<0x141>(v);  // the other four of eight
    if constexpr (LANES >= 16)
        v = dpp_add_f32<0x140>(v);  // the other eight of sixteen
    if constexpr (LANES >= 32)
        v = add_across<16>(v);
    return v;
}
// over the teams of a wave, lane by lane
template <int LANES>
__device__ __forceinline__ float teams_sum(float v)
{
    // rows of 16 turned by 8, 4, 2 and 1
    if constexpr (LANES <= 8)
        v = dpp_add_f32<0x128>(v);
    if constexpr (LANES <= 4)
        v = dpp_add_f32<0x124>(v);
    if constexpr (LANES <= 2)
        v = dpp_add_f32<0x122>(v);
    if constexpr (LANES <= 1)
        v = dpp_add_f32<0x121>(v);
    if constexpr (LANES <= 16)
        v = add_across<16>(v);
    if constexpr (LANES <= 32)
        v = add_across<32>(v);
    return v;
}

// x becomes xhat.  Squares whose sum leaves fp32 (beyond 2^100, or, without an eps that covers them, below 2^-80) are taken of values
// moved by a power of two.
template <int LANES, int PER>
__device__ __forceinline__ float heads_normalise(float (&a)[PER], float (&b)[PER], float per_dim, float eps)
{
    auto squares = [&] {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < PER; ++e)
            ss = __builtin_fmaf(a[e], a[e], __builtin_fmaf(b[e], b[e], ss));
        return team_sum<LANES>(ss);
    };
    const float ss = squares();
    float rstd = __builtin_amdgcn_rsqf(__builtin_fmaf(ss, per_dim, eps)), moved = 1.0f;
    if (!(ss < 0x1p100f) || (ss < 0x1p-80f && eps < 0x1p-80f)) {
        moved = ss < 1.0f ? 0x1p100f : 0x1p-90f;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            a[e] *= moved;
            b[e] *= moved;
        }
        rstd = (float)(1.0 / __builtin_sqrt((double)squares() * per_dim + (double)eps * moved * moved));
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        a[e] *= rstd;
        b[e] *= rstd;
    }
    return rstd * moved;
}

enum HeadsMode { kHeadsRotary, kHeadsNorm, kHeadsGrad };

// ONCE: large calls; what is read is read past the caches.
template <typename LANE, int LANES, int MODE, bool ONCE>
__global__ __launch_bounds__(kHeadsThreads, MODE != kHeadsGrad ? 4 : LANE::CHUNKS < 8 ? 3 : 2) void heads_kernel(HeadsDev g)
{
    constexpr int PER = LANE::PER, TEAMS = kHeadsThreads / LANES;
    __shared__ float2 angles[kHeadsAngles];
    __shared__ int padding[kHeadsTokens];
    const bool second = (int)blockIdx.x >= g.side[0].blocks;
    const HeadsSide &side = g.side[second];
    const int block = (int)blockIdx.x - (second ? g.side[0].blocks : 0), split = block % side.splits;
    const int h0 = split * side.block_heads, nh = min(side.block_heads, side.heads - h0);
    const int64_t t0 = (int64_t)(block / side.splits) * side.block_tokens, step = (int64_t)(side.blocks / side.splits) * side.block_tokens;
    const int tid = threadIdx.x, team = tid / LANES, half = g.rot >> 1;
    const LANE lane(tid & (LANES - 1), g.dim, g.rot);
    const float per_half = half != 0 ? 1.0f / (float)half : 0.0f, per_head = 1.0f / (float)nh, per_dim = 1.0f / (float)g.dim;

    float ga[PER], gb[PER];
    if constexpr (MODE != kHeadsRotary) {
        if (side.gain != nullptr) {
            lane.widen(lane.template fetch<false>(side.gain), ga, gb);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                ga[e] = gb[e] = 1.0f;
        }
    }
    float sa[PER], sb[PER];  // dgain of what the lane has seen
    if constexpr (MODE == kHeadsGrad)
#pragma unroll
        for (int e = 0; e < PER; ++e)
            sa[e] = sb[e] = 0.0f;

    for (int64_t t = t0; t < g.tokens; t += step) {
        const int nt = (int)min((int64_t)side.block_tokens, g.tokens - t);
        const uint16_t *x0 = side.x + t * side.x_token + (int64_t)h0 * side.x_head, *dy0 = side.dy + t * side.dy_token + (int64_t)h0 * side.dy_head;
        uint16_t *y0 = side.y + t * side.y_token + (int64_t)h0 * side.y_head;
        // an item is a head of a token; its heads are fetched one round ahead (padding too, which is there)
        auto token_of = [&](int item) { return (int)(((float)item + 0.5f) * per_head); };
        auto place = [&](int item, int64_t token, int64_t head) {
            const int ti = token_of(item);
            return (uint64_t)(uint32_t)ti * (uint64_t)token + (uint64_t)(uint32_t)(item - ti * nh) * (uint64_t)head;
        };
        typename LANE::Raw x{}, dy{};
        auto fetch = [&](int item) {
            x = lane.template fetch<ONCE>(x0 + place(item, side.x_token, side.x_head));
            if constexpr (MODE == kHeadsGrad)
                dy = lane.template fetch<ONCE>(dy0 + place(item, side.dy_token, side.dy_head));
        };
        const int items = nt * nh;
        if (team < items)
            fetch(team);
        if (t != t0)
            __syncthreads();
        for (int i = tid; i < nt * half; i += kHeadsThreads) {
            const int ti = (int)(((float)i + 0.5f) * per_half), p = i - ti * half;
            const int64_t position = g.positions[t + ti];
            if (p == 0)
                padding[ti] = position < 0;
            // in turns: the fraction is exact to the product's own rounding, 2^-52 of the turns
            const double turns = (double)position * g.freqs[p] * 0.15915494309189533577;
            float sine, cosine;
            sincospif(2.0f * (float)(turns - __builtin_rint(turns)), &sine, &cosine);
            angles[i] = make_float2(cosine * g.scale, sine * g.sign * g.scale);
        }
        if (half != 0)
            __syncthreads();
        for (int item = team; item < items; item += TEAMS) {
            const int ti = token_of(item);
            const float2 *cs = angles + ti * half;
            float a[PER], b[PER], da[PER], db[PER];
            lane.widen(x, a, b);
            if constexpr (MODE == kHeadsGrad)
                lane.widen(dy, da, db);
            if (item + TEAMS < items)
                fetch(item + TEAMS);
            if (half != 0 && padding[ti])
                continue;
            auto turn = [&](float (&a)[PER], float (&b)[PER]) {
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (lane.rotates(e)) {
                        const float2 c = cs[lane.angle(e)];
                        const float u = a[e] * c.x - b[e] * c.y, v = b[e] * c.x + a[e] * c.y;
                        a[e] = u;
                        b[e] = v;
                    }
            };
            if constexpr (MODE == kHeadsNorm) {
                heads_normalise<LANES>(a, b, per_dim, g.eps);
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    a[e] *= ga[e];
                    b[e] *= gb[e];
                }
            }
            if constexpr (MODE != kHeadsGrad) {
                turn(a, b);
            } else {
                turn(da, db);
                const float rstd = heads_normalise<LANES>(a, b, per_dim, g.eps);
                float dot = 0.0f;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    sa[e] = __builtin_fmaf(da[e], a[e], sa[e]);
                    sb[e] = __builtin_fmaf(db[e], b[e], sb[e]);
                    da[e] *= ga[e];
                    db[e] *= gb[e];
                    dot = __builtin_fmaf(da[e], a[e], __builtin_fmaf(db[e], b[e], dot));
                }
                dot = team_sum<LANES>(dot) * per_dim;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    a[e] = rstd * __builtin_fmaf(-a[e], dot, da[e]);
                    b[e] = rstd * __builtin_fmaf(-b[e], dot, db[e]);
                }
            }
            lane.store(y0 + place(item, side.y_token, side.y_head), a, b);
        }
    }
    if (MODE == kHeadsGrad && g.partials != nullptr) {
        // over the teams of a wave, then, column by column, over the waves
        constexpr int WAVES = kHeadsThreads / kWave;
        float *sums = (float *)angles;
        static_assert(WAVES * kHeadsMaxDim <= 2 * kHeadsAngles, "the angles' room");
        const int wave = tid / kWave;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            sa[e] = teams_sum<LANES>(sa[e]);
            sb[e] = teams_sum<LANES>(sb[e]);
        }
        __syncthreads();
        if ((tid & (kWave - 1)) < LANES)
#pragma unroll
            for (int e = 0; e < 2 * PER; ++e) {
                const int c = lane.column(e >> 1, e & 1);
                if (c >= 0)
                    sums[wave * kHeadsMaxDim + c] = e & 1 ? sb[e >> 1] : sa[e >> 1];
            }
        __syncthreads();
        for (int c = tid; c < g.dim; c += kHeadsThreads) {
            float s = sums[c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
                s += sums[w * kHeadsMaxDim + c];
            g.partials[(int64_t)blockIdx.x * g.dim + c] = s;
        }
    }
}

// dgain: the workgroups' rows, 16 columns a workgroup, added in a fixed order
__global__ __launch_bounds__(256) void heads_gain_kernel(const float *__restrict__ partials, int rows0, int rows1, int dim,
                                                         float *dgain0, float *dgain1)
{
    __shared__ float red[16][17];
    const bool second = blockIdx.y != 0;
    float *out = second ? dgain1 : dgain0;
    const int from = second ? rows0 : 0, to = second ? rows0 + rows1 : rows0;
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
    if (out == nullptr)
        return;
    float s = 0.0f;
    if (c < dim)
#pragma unroll 8
        for (int i = from + r; i < to; i += 16)
            s += partials[(int64_t)i * dim + c];
    red[r][threadIdx.x & 15] = s;
    __syncthreads();
    if (r == 0 && c < dim) {
#pragma unroll
        for (int i = 1; i < 16; ++i)
            s += red[i][threadIdx.x];
        out[c] = s;
    }
}

// ---- host side
// Rotation, from so many bytes on, by teams whose loads cover whole lines: 16384x32 of 128 53 us, read past the caches 50; of 64, whose
// pieces of a line are fetched by two loads, 53 and 55; the norm 55 both ways, gradients 83 and 88.
constexpr int64_t kHeadsOnceBytes = 128 << 20;
constexpr int kHeadsBlockHeads = 2048;  // (a workgroup divides its items by them in fp32)
constexpr int kHeadsGradBlocks = 768;  // workgroups of the gradients, three a CU
// Heads of a team at a time.  us, 1 / 2 / 4 / 8: rotation of 16384x32 of 128 53 / 50 / 52 / 57, 4096x40 of 128 17.8 / 16.5 / 16.6 / -; norm of
// 16384x64 of 64 68 / 56 / 55 / 64
constexpr int kHeadsRounds = 4, kHeadsRoundsRotary = 2;

// a row of dgain for each workgroup: each side has its share of them, one at least
int64_t heads_grad_bytes(int64_t tokens, int64_t heads, int64_t dim)
{
    return std::min<int64_t>(tokens * heads, kHeadsGradBlocks + 1) * dim * 4;
}

// items: heads at a time; most: workgroups at most (a side has a 768th of all heads for each, so that its heads in that many parts
// are 512 at a time at most)
static void heads_share(HeadsSide &s, int64_t tokens, int64_t items, int64_t at_once, int64_t most)
{
    s.block_heads = (int)std::min<int64_t>(s.heads, std::max(std::min<int64_t>(items, kHeadsBlockHeads), (s.heads + most - 1) / most));
    s.block_tokens = (int)std::min<int64_t>({tokens, at_once, (items + s.block_heads - 1) / s.block_heads});
    s.splits = (s.heads + s.block_heads - 1) / s.block_heads;
    const int64_t rows = (tokens + s.block_tokens - 1) / s.block_tokens;
    s.blocks = (int)(s.splits * std::min(rows, std::max<int64_t>(1, most / s.splits)));
}

template <bool PAIRS, int V, int LANES>
static hipError_t launch_lanes(HeadsDev &g, int mode, int sides, hipStream_t s)
{
    typedef HeadsLane<PAIRS, V, LANES> LANE;
    constexpr int TEAMS = kHeadsThreads / LANES;
    const int half = g.rot / 2;
    const int64_t at_once = half != 0 ? std::min(kHeadsTokens, kHeadsAngles / half) : kHeadsTokens;
    int64_t all = 0;
    for (int i = 0; i < sides; ++i)
        all += g.tokens * g.side[i].heads;
    for (int i = 0; i < sides; ++i) {
        const int64_t mine = g.tokens * g.side[i].heads;
        const int64_t items = std::min<int64_t>((mode == kHeadsRotary ? kHeadsRoundsRotary : kHeadsRounds) * TEAMS, std::max<int64_t>(TEAMS, mine / 1024));
        heads_share(g.side[i], g.tokens, items, at_once, mode == kHeadsGrad ? std::max<int64_t>(1, kHeadsGradBlocks * mine / all) : (int64_t)1 << 31);
    }
    const dim3 grid((unsigned)(g.side[0].blocks + g.side[1].blocks)), block(kHeadsThreads);
    constexpr bool USUAL = V == 8 && LANES >= 8 && LANES <= 16;
    if (mode == kHeadsRotary && USUAL && all * g.dim * 4 >= kHeadsOnceBytes)
        hipLaunchKernelGGL((heads_kernel<LANE, LANES, kHeadsRotary, USUAL>), grid, block, 0, s, g);
    else if (mode == kHeadsRotary)
        hipLaunchKernelGGL((heads_kernel<LANE, LANES, kHeadsRotary, false>), grid, block, 0, s, g);
    else if (mode == kHeadsNorm)
        hipLaunchKernelGGL((heads_kernel<LANE, LANES, kHeadsNorm, false>), grid, block, 0, s, g);
    else
        hipLaunchKernelGGL((heads_kernel<LANE, LANES, kHeadsGrad, false>), grid, block, 0, s, g);
    return hipGetLastError();
}

template <bool PAIRS, int V>
static hipError_t launch_width(HeadsDev &g, int mode, int sides, hipStream_t s)
{
    const int lanes = (g.dim + 15) / 16;
    if constexpr (V == 8) {
        if (lanes <= 1)
            return launch_lanes<PAIRS, V, 1>(g, mode, sides, s);
        if (lanes <= 2)
            return launch_lanes<PAIRS, V, 2>(g, mode, sides, s);
    }
    if (lanes <= 4)
        return launch_lanes<PAIRS, V, 4>(g, mode, sides, s);
    if (lanes <= 8)
        return launch_lanes<PAIRS, V, 8>(g, mode, sides, s);
    if (lanes <= 16)
        return launch_lanes<PAIRS, V, 16>(g, mode, sides, s);
    return launch_lanes<PAIRS, V, 32>(g, mode, sides, s);
}

// chunks of V pairs, where both members' chunks and what is left are whole ones
template <bool PAIRS>
static hipError_t launch_layout(HeadsDev &g, int mode, int sides, hipStream_t s)
{
    const int pairs = g.rot / 2;
    if (pairs % 8 == 0 && g.dim % 8 == 0)
        return launch_width<PAIRS, 8>(g, mode, sides, s);
    return pairs % 2 == 0 && g.dim % 2 == 0 ? launch_width<PAIRS, 2>(g, mode, sides, s) : launch_width<PAIRS, 1>(g, mode, sides, s);
}

hipError_t launch_heads(const HeadsCall &c, int mode, hipStream_t s)
{
    HeadsDev g{};
    g.tokens = c.tokens;
    g.dim = c.dim;
    g.rot = c.rot;
    g.positions = c.positions;
    g.freqs = c.freqs;
    g.scale = c.scale;
    g.eps = c.eps;
    g.sign = c.transpose || mode == kHeadsGrad ? -1.0f : 1.0f;
    g.partials = c.partials;
    for (int i = 0; i < c.sides; ++i) {
        const HeadsCallSide &f = c.side[i];
        HeadsSide &t = g.side[i];
        t.x = (const uint16_t *)f.x;
        t.dy = (const uint16_t *)f.dy;
        t.gain = (const uint16_t *)f.gain;
        t.y = (uint16_t *)f.y;
        t.heads = f.heads;
        // a stride that no second token or head is reached by says nothing
        auto stride = [](int64_t v, int64_t n) { return n > 1 ? v : 0; };
        t.x_token = stride(f.x_token, c.tokens);
        t.x_head = stride(f.x_head, f.heads);
        t.dy_token = stride(f.dy_token, c.tokens);
        t.dy_head = stride(f.dy_head, f.heads);
        t.y_token = stride(f.y_token, c.tokens);
        t.y_head = stride(f.y_head, f.heads);
    }
    const hipError_t e = c.pairs ? launch_layout<true>(g, mode, c.sides, s) : launch_layout<false>(g, mode, c.sides, s);
    if (e != hipSuccess || mode != kHeadsGrad || (c.side[0].dgain == nullptr && c.side[1].dgain == nullptr))
        return e;
    hipLaunchKernelGGL(heads_gain_kernel, dim3((unsigned)((c.dim + 15) / 16), (unsigned)c.sides), dim3(256), 0, s, g.partials,
                       g.side[0].blocks, g.side[1].blocks, c.dim, c.side[0].dgain, c.side[1].dgain);
    return hipGetLastError();
}

hipError_t launch_rotary(const HeadsCall &c, hipStream_t s) { return launch_heads(c, kHeadsRotary, s); }
hipError_t launch_head_norm(const HeadsCall &c, hipStream_t s) { return launch_heads(c, kHeadsNorm, s); }
hipError_t launch_head_norm_grad(const HeadsCall &c, hipStream_t s) { return launch_heads(c, kHeadsGrad, s); }

}  // namespace tweo
