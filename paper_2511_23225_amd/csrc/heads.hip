// Heads of queries and keys (gfx950): rotation by position, norm of each head with the rotation behind it, and the norm's gradients.
//
//   angle  = position * freq (fp64), taken modulo a turn before it becomes fp32
//   R      : (a, b) -> scale * (a cos - b sin, b cos + a sin) on the pairs of the first `rot` values of a head, the others as they are
//   rotary : y = R x, or (transposed, the gradient) R^T x
//   norm   : xhat = x * rstd, rstd = 1 / sqrt(mean(x^2) + eps), y = R (xhat * gain)
//   grad   : d = R^T dy, w = d * gain, dx = rstd * (w - xhat * mean(w * xhat)), dgain = sum over tokens and heads of d * xhat
//
// A head belongs to a team of 1 to 32 lanes (a power of two, 16 values each) that hold both members of a pair in one lane, in 16-byte pieces, which
// overlap where width and turned part are no whole ones.  The angles of a workgroup's tokens are worked out once, one a thread, into LDS and serve
// all heads; nothing else is shared, so memory bounds the large calls: 16384 tokens of 32 heads of 128, rotation 49 us (5.5 TB/s, a copy's
// rate and more), 64 of 64, norm 55 and gradients 81.5 (78.5 and the joining of dgain's rows).
#include <algorithm>
#include <type_traits>
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

// ---- where a lane's eight pairs lie.  a, b: the members of a pair, or of what is not turned, what lies there.
typedef uint32_t HeadsPiece __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any even address

template <bool ONCE>
__device__ __forceinline__ void fetch_piece(const uint16_t *p, int at, uint32_t *w)
{
    HeadsPiece v = {0, 0, 0, 0};
    if (at >= 0)
        v = ONCE ? __builtin_nontemporal_load((const HeadsPiece *)(p + at)) : *(const HeadsPiece *)(p + at);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        w[k] = v[k];
}

// Sixteen elements in two pieces: first and second members (halves), or pairs one behind the other, of the turned part, then of what is left.
// OVER: parts that are no whole pieces.  A part's last pieces then end where the part does and hold some elements that those in front of them
// hold too: both lanes come to the same results and store them, one counts them in sums.  Less than sixteen elements that are left are the end of
// pieces whose other elements belong to the turned part; they are stored one by one.  us, 16384x32 of 100, rotation / norm / gradients: 51 / 54 /
// 93, in words (pairs l, l + LANES, ..) 66 / 66 / 84; of 98 with 66 turned 50 / 57 / 73 (in pairs), element by element 84 / 91 / 169.
template <bool PAIRS, int LANES, bool OVER>
struct HeadsPieces {
    static constexpr int PER = 8;
    static constexpr bool FAST = !OVER;
    int at_a, at_b;  // first elements, -1: none
    int pair0;       // first pair's number
    int from_a, from_b;  // OVER: the pairs, by member, from which on they count
    bool turns, part;    // part: only what counts is stored
    __device__ __forceinline__ HeadsPieces(int l, int dim, int rot)
    {
        if constexpr (!OVER) {
            const int lanes = rot >> 4;
            turns = l < lanes;
            at_a = turns && !PAIRS ? 8 * l : 16 * l;
            at_b = turns && !PAIRS ? 8 * (l + lanes) : at_a + 8;
            at_a = at_a < dim ? at_a : -1;
            at_b = at_b < dim ? at_b : -1;
            pair0 = 8 * l;
            from_a = from_b = 0;
            part = false;
        } else {
            const int lanes = (rot + 15) >> 4, left = dim - rot;
            turns = l < lanes;
            // sixteen elements from `at` of a part of `len` (its first, `first`), `shift` of them counted by the lane before
            const int first = turns ? 0 : rot, len = turns ? rot : left, at = 16 * (turns ? l : l - lanes);
            const bool none = at >= len;
            const int start = at + 16 <= len ? at : len - 16, shift = none ? 16 : at - start;
            part = !turns && len < 16;  // (start is negative: into the turned part)
            if (turns && !PAIRS) {  // members of eight pairs, from pair start / 2 on; shift / 2 pairs too many
                at_a = start >> 1;
                at_b = at_a + (rot >> 1);
                from_a = from_b = shift >> 1;
            } else {
                at_a = first + start;
                at_b = at_a + 8;
                from_a = PAIRS ? (shift + 1) >> 1 : shift;
                from_b = PAIRS ? shift >> 1 : shift - 8;
            }
            if (none)
                at_a = at_b = -1;
            pair0 = start >> 1;
        }
    }
    __device__ __forceinline__ bool rotates(int) const { return turns; }
    __device__ __forceinline__ int angle(int e) const { return pair0 + e; }
    __device__ __forceinline__ bool counts(int e, bool second) const { return !OVER || e >= (second ? from_b : from_a); }
    // a column of the head that counts, or -1
    __device__ __forceinline__ int column(int e, bool second) const
    {
        const int pos = PAIRS ? 2 * e + second : second ? 8 + e : e, from = pos < 8 ? at_a : at_b;
        return from < 0 || !counts(e, second) ? -1 : from + (pos & 7);
    }
    struct Raw {
        uint32_t w[8];
    };
    template <bool ONCE>
    __device__ __forceinline__ Raw fetch(const uint16_t *p) const
    {
        Raw r;
        fetch_piece<ONCE>(p, at_a, r.w);
        fetch_piece<ONCE>(p, at_b, r.w + 4);
        return r;
    }
    __device__ __forceinline__ void widen(const Raw &r, float (&a)[PER], float (&b)[PER]) const
    {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const uint32_t wa = r.w[PAIRS ? e : e >> 1], wb = r.w[PAIRS ? e : 4 + (e >> 1)];
            a[e] = !PAIRS && (e & 1) ? bf16hi_to_f32(wa) : bf16lo_to_f32(wa);
            b[e] = PAIRS || (e & 1) ? bf16hi_to_f32(wb) : bf16lo_to_f32(wb);
        }
    }
    __device__ __forceinline__ void store(uint16_t *p, const float (&a)[PER], const float (&b)[PER]) const
    {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            w[k] = PAIRS ? pack_bf16x2(a[k], b[k]) : k < 4 ? pack_bf16x2(a[2 * (k & 3)], a[2 * (k & 3) + 1]) : pack_bf16x2(b[2 * (k & 3)], b[2 * (k & 3) + 1]);
        if (OVER && part) {
#pragma unroll
            for (int e = 0; e < 2 * PER; ++e) {
                const int c = column(e >> 1, e & 1), k = PAIRS ? e >> 1 : (e & 1) * 4 + (e >> 2);
                if (c >= 0)
                    p[c] = (uint16_t)(PAIRS ? w[k] >> (16 * (e & 1)) : w[k] >> (16 * ((e >> 1) & 1)));
            }
            return;
        }
        if (at_a >= 0)
            *(HeadsPiece *)(p + at_a) = HeadsPiece{w[0], w[1], w[2], w[3]};
        if (at_b >= 0)
            *(HeadsPiece *)(p + at_b) = HeadsPiece{w[4], w[5], w[6], w[7]};
    }
};

// Element by element, pairs l, l + LANES, ..: heads of less than sixteen elements, or with less than sixteen turned, and the widest that are no whole pieces
template <bool PAIRS, int LANES>
struct HeadsElements {
    static constexpr int PER = 8;
    static constexpr bool FAST = false;
    int l, dim, half;
    __device__ __forceinline__ HeadsElements(int l_, int dim_, int rot) : l(l_), dim(dim_), half(rot >> 1) {}
    __device__ __forceinline__ bool rotates(int e) const { return angle(e) < half; }
    __device__ __forceinline__ int angle(int e) const { return l + LANES * e; }
    __device__ __forceinline__ bool counts(int, bool) const { return true; }
    __device__ __forceinline__ int column(int e, bool second) const
    {
        const int p = angle(e), c = PAIRS || p >= half ? 2 * p + second : second ? p + half : p;
        return c < dim ? c : -1;
    }
    struct Raw {
        uint32_t w[2 * PER];
    };
    template <bool ONCE>
    __device__ __forceinline__ Raw fetch(const uint16_t *p) const
    {
        Raw r;
#pragma unroll
        for (int e = 0; e < 2 * PER; ++e) {
            const int c = column(e >> 1, e & 1);
            r.w[e] = c >= 0 ? (uint32_t)p[c] << 16 : 0u;
        }
        return r;
    }
    __device__ __forceinline__ void widen(const Raw &r, float (&a)[PER], float (&b)[PER]) const
    {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            a[e] = bits_to_f32(r.w[2 * e]);
            b[e] = bits_to_f32(r.w[2 * e + 1]);
        }
    }
    __device__ __forceinline__ void store(uint16_t *p, const float (&a)[PER], const float (&b)[PER]) const
    {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const uint32_t d = pack_bf16x2(a[e], b[e]);
            const int i = column(e, false), j = column(e, true);
            if (i >= 0)
                p[i] = (uint16_t)d;
            if (j >= 0)
                p[j] = (uint16_t)(d >> 16);
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
template <int LANES, int PER, typename LANE>
__device__ __forceinline__ float heads_normalise(const LANE &lane, float (&a)[PER], float (&b)[PER], float per_dim, float eps)
{
    auto squares = [&] {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const float u = lane.counts(e, false) ? a[e] : 0.0f, v = lane.counts(e, true) ? b[e] : 0.0f;
            ss = __builtin_fmaf(u, u, __builtin_fmaf(v, v, ss));
        }
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
__global__ __launch_bounds__(kHeadsThreads, MODE != kHeadsGrad ? 4 : LANE::FAST ? 3 : 2) void heads_kernel(HeadsDev g)
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
                        // (spelled out: a value that two lanes hold has to come out the same in both)
                        const float u = __builtin_fmaf(a[e], c.x, -(b[e] * c.y)), v = __builtin_fmaf(b[e], c.x, a[e] * c.y);
                        a[e] = u;
                        b[e] = v;
                    }
            };
            if constexpr (MODE == kHeadsNorm) {
                heads_normalise<LANES>(lane, a, b, per_dim, g.eps);
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
                const float rstd = heads_normalise<LANES>(lane, a, b, per_dim, g.eps);
                float dot = 0.0f;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    sa[e] = __builtin_fmaf(da[e], a[e], sa[e]);
                    sb[e] = __builtin_fmaf(db[e], b[e], sb[e]);
                    da[e] *= ga[e];
                    db[e] *= gb[e];
                    const float u = lane.counts(e, false) ? da[e] : 0.0f, v = lane.counts(e, true) ? db[e] : 0.0f;
                    dot = __builtin_fmaf(u, a[e], __builtin_fmaf(v, b[e], dot));
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
constexpr int64_t kHeadsMostBlocks = (int64_t)1 << 22;  // of a group: a launch holds less than 2^32 threads
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

template <typename LANE, int LANES>
static hipError_t launch_lanes(HeadsDev &g, int mode, int sides, hipStream_t s)
{
    constexpr int TEAMS = kHeadsThreads / LANES;
    const int half = g.rot / 2;
    const int64_t at_once = half != 0 ? std::min(kHeadsTokens, kHeadsAngles / half) : kHeadsTokens;
    int64_t all = 0;
    for (int i = 0; i < sides; ++i)
        all += g.tokens * g.side[i].heads;
    for (int i = 0; i < sides; ++i) {
        const int64_t mine = g.tokens * g.side[i].heads;
        const int64_t items = std::min<int64_t>((mode == kHeadsRotary ? kHeadsRoundsRotary : kHeadsRounds) * TEAMS, std::max<int64_t>(TEAMS, mine / 1024));
        heads_share(g.side[i], g.tokens, items, at_once, mode == kHeadsGrad ? std::max<int64_t>(1, kHeadsGradBlocks * mine / all) : kHeadsMostBlocks);
    }
    const dim3 grid((unsigned)(g.side[0].blocks + g.side[1].blocks)), block(kHeadsThreads);
    constexpr bool USUAL = LANE::FAST && LANES >= 8 && LANES <= 16;
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

enum HeadsWidth { kHeadsWhole, kHeadsOver, kHeadsElement };
template <bool PAIRS, int WIDTH>
static hipError_t launch_width(HeadsDev &g, int mode, int sides, int lanes, hipStream_t s)
{
    auto launch = [&](auto lanes_c) {
        constexpr int LANES = decltype(lanes_c)::value;
        if constexpr (WIDTH == kHeadsElement)
            return launch_lanes<HeadsElements<PAIRS, LANES>, LANES>(g, mode, sides, s);
        else
            return launch_lanes<HeadsPieces<PAIRS, LANES, WIDTH == kHeadsOver>, LANES>(g, mode, sides, s);
    };
    if constexpr (WIDTH == kHeadsWhole)
        if (lanes <= 1)
            return launch(std::integral_constant<int, 1>{});
    if constexpr (WIDTH != kHeadsElement)
        if (lanes <= 2)
            return launch(std::integral_constant<int, 2>{});
    if (lanes <= 4)
        return launch(std::integral_constant<int, 4>{});
    if (lanes <= 8)
        return launch(std::integral_constant<int, 8>{});
    if (lanes <= 16)
        return launch(std::integral_constant<int, 16>{});
    return launch(std::integral_constant<int, 32>{});
}

template <bool PAIRS>
static hipError_t launch_layout(HeadsDev &g, int mode, int sides, hipStream_t s)
{
    const int left = g.dim - g.rot, over = (g.rot + 15) / 16 + (left + 15) / 16;
    if (g.rot % 16 == 0 && g.dim % 8 == 0)
        return launch_width<PAIRS, kHeadsWhole>(g, mode, sides, (g.dim + 15) / 16, s);
    if (g.dim >= 16 && (g.rot == 0 || g.rot >= 16) && over <= 32)
        return launch_width<PAIRS, kHeadsOver>(g, mode, sides, over, s);
    return launch_width<PAIRS, kHeadsElement>(g, mode, sides, (g.dim + 15) / 16, s);
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
