// LayerNorm to bf16, forward and backward.  Rows of any length; gfx950 only.
#include <algorithm>
#include "kernels.h"
#include "layernorm.h"

namespace tweo {

namespace {

// ---------------------------------------------------------------------------
// A row is worked on by a team of T waves; lane l of the team holds the 16-byte pieces (eight elements) l, l + 64 T, ... of it,
// P of them, in registers.  RAGGED: cols is no multiple of eight, so rows start at any even address and their last piece is short.

typedef uint32_t loose_u4 __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any even address

template <bool RAGGED>
struct Row {
    int cols, pieces;
    __device__ __forceinline__ explicit Row(int cols_) : cols(cols_), pieces(RAGGED ? (cols_ + 7) >> 3 : cols_ >> 3) {}
    // elements of piece i
    __device__ __forceinline__ int count(int i) const
    {
        if constexpr (!RAGGED)
            return i < pieces ? 8 : 0;
        const int left = cols - 8 * i;
        return left < 0 ? 0 : left < 8 ? left : 8;
    }
    // piece i of the row at p, with zeros behind its end; a lane without a piece gets one of the row's (aligned rows: with a
    // branch around each load the compiler waits for one before it issues the next) or zeros
    __device__ __forceinline__ uint4 load(const uint16_t *p, int i) const
    {
        if constexpr (!RAGGED) {
            const int last = pieces - 1, j = i < last ? i : last;
            return *(const uint4 *)((const uint8_t *)p + (uint64_t)((uint32_t)j * 16u));
        }
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        const int n = count(i);
        if (n == 8) {
            const loose_u4 l = *(const loose_u4 *)(p + 8 * (int64_t)i);
            v = make_uint4(l[0], l[1], l[2], l[3]);
        } else if (n > 0) {
            uint32_t e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                e[k] = k < n ? p[8 * (int64_t)i + k] : 0u;
            v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
        return v;
    }
    __device__ __forceinline__ void store(uint16_t *p, int i, uint4 v) const
    {
        if constexpr (!RAGGED) {
            if (i < pieces)
                *(uint4 *)((uint8_t *)p + (uint64_t)((uint32_t)i * 16u)) = v;
            return;
        }
        const int n = count(i);
        if (n == 8) {
            *(loose_u4 *)(p + 8 * (int64_t)i) = loose_u4{v.x, v.y, v.z, v.w};
        } else if (n > 0) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 7; ++k)
                if (k < n)
                    p[8 * (int64_t)i + k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
        }
    }
};

// sum of squared differences of the first n elements of a piece
template <bool RAGGED>
__device__ __forceinline__ double squares(uint4 v, double mean, int n)
{
    if constexpr (!RAGGED) {
        const double t = sumsq8_f64(v, mean);
        return n > 0 ? t : 0.0;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const double d0 = (double)bf16lo_to_f32(w[k]) - mean, d1 = (double)bf16hi_to_f32(w[k]) - mean;
        s += (2 * k < n ? d0 * d0 : 0.0) + (2 * k + 1 < n ? d1 * d1 : 0.0);
    }
    return s;
}

// Sum over the T waves of a team: of each wave through DPP, then through LDS, added in the waves' order by all of them.  `red`: the
// T words of this team for this sum, which are free again two barriers later.
template <int T>
__device__ __forceinline__ double team_sum(double v, double *red, int wave)
{
    v = wave_sum_f64(v);
    if constexpr (T > 1) {
        if ((threadIdx.x & (kWave - 1)) == 0)
            red[wave] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < T; ++w)
            v += red[w];
    }
    return v;
}

// ---------------------------------------------------------------------------
// Forward: y = (h - mu) / sqrt(var + eps) * gamma + beta, h = x or bf16(x + residual).  One read of a row (2 B an element, 4 with a
// residual), one write (2, 4): mean and squared differences are taken of the registers, in fp64 as in the pass in front of the
// FP8 cast, whose stored activation this one's equals bit for bit.
struct LnFwdArgs {
    const uint16_t *x, *res, *gamma, *beta;
    uint16_t *h, *y;
    double *stats;
    int64_t rows;
    int cols;
    double eps;
};

template <int T>
constexpr int kFwdWaves = T > 4 ? T : 4;

template <int T, int P, bool RES, bool RAGGED>
__global__ __launch_bounds__(kFwdWaves<T> *kWave) void ln_fwd_kernel(LnFwdArgs a)
{
    constexpr int WAVES = kFwdWaves<T>, TEAMS = WAVES / T;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), team = wave / T;
    const int lane = (int)threadIdx.x - team * T * kWave;
    const Row<RAGGED> row(a.cols);
    const double n = (double)a.cols;
    __shared__ double red[2][WAVES];
    for (int64_t r0 = (int64_t)blockIdx.x * TEAMS; r0 < a.rows; r0 += (int64_t)gridDim.x * TEAMS) {
        // a team without a row goes through the last one's sums with the others (barriers) and stores nothing
        const bool mine = r0 + team < a.rows;
        const int64_t r = mine ? r0 + team : a.rows - 1;
        if (T == 1 && !mine)
            return;
        uint4 c[P];
        double s = 0.0;
#pragma unroll
        for (int u = 0; u < P; ++u)
            c[u] = row.load(a.x + r * a.cols, lane + u * T * kWave);
        if constexpr (RES) {
            uint4 d[P];
#pragma unroll
            for (int u = 0; u < P; ++u)
                d[u] = row.load(a.res + r * a.cols, lane + u * T * kWave);
#pragma unroll
            for (int u = 0; u < P; ++u) {
                c[u] = add_bf16x8(c[u], d[u]);
                if (mine)
                    row.store(a.h + r * a.cols, lane + u * T * kWave, c[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const double t = sum8_f64(c[u]);
            s += row.count(lane + u * T * kWave) > 0 ? t : 0.0;
        }
        const double mean = team_sum<T>(s, &red[0][team * T], wave - team * T) / n;
        double ss = 0.0;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            // the packed form is what stays in registers, not its widened values
            asm volatile("" : "+v"(c[u].x), "+v"(c[u].y), "+v"(c[u].z), "+v"(c[u].w));
            ss += squares<RAGGED>(c[u], mean, row.count(lane + u * T * kWave));
        }
        const double rstd = 1.0 / __builtin_sqrt(team_sum<T>(ss, &red[1][team * T], wave - team * T) / n + a.eps);
        if (!mine)
            continue;
        if (a.stats != nullptr && lane == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
#pragma unroll
        for (int u = 0; u < P; ++u) {
            asm volatile("" : "+v"(c[u].x), "+v"(c[u].y), "+v"(c[u].z), "+v"(c[u].w));
            const int i = lane + u * T * kWave;
            double g[8], b[8];
            widen8(row.load(a.gamma, i), g);
            widen8(a.beta != nullptr ? row.load(a.beta, i) : make_uint4(0u, 0u, 0u, 0u), b);
            row.store(a.y + r * a.cols, i, ln_vec(c[u], mean, rstd, g, b, a.beta != nullptr));
        }
    }
}

// Rows longer than a team's registers: a workgroup a row, which it reads three times (from the caches when they hold it).
constexpr int kWideThreads = 512;

template <bool RES, bool RAGGED>
__global__ __launch_bounds__(kWideThreads) void ln_fwd_wide_kernel(LnFwdArgs a)
{
    constexpr int T = kWideThreads / kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Row<RAGGED> row(a.cols);
    const double n = (double)a.cols;
    __shared__ double red[2][T];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        double s = 0.0;
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads) {
            uint4 v = row.load(a.x + r * a.cols, i);
            if constexpr (RES) {
                v = add_bf16x8(v, row.load(a.res + r * a.cols, i));
                row.store(a.h + r * a.cols, i, v);
            }
            s += sum8_f64(v);
        }
        // h may be x or the residual itself: what this thread has stored is read back, not formed again
        const uint16_t *h = RES ? a.h : a.x;
        const double mean = team_sum<T>(s, red[0], wave) / n;
        double ss = 0.0;
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads)
            ss += squares<RAGGED>(row.load(h + r * a.cols, i), mean, row.count(i));
        const double rstd = 1.0 / __builtin_sqrt(team_sum<T>(ss, red[1], wave) / n + a.eps);
        if (a.stats != nullptr && threadIdx.x == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads) {
            double g[8], b[8];
            widen8(row.load(a.gamma, i), g);
            widen8(a.beta != nullptr ? row.load(a.beta, i) : make_uint4(0u, 0u, 0u, 0u), b);
            row.store(a.y + r * a.cols, i, ln_vec(row.load(h + r * a.cols, i), mean, rstd, g, b, a.beta != nullptr));
        }
    }
}

constexpr int kCus = 256;  // of an MI355X; a device with more or fewer runs the same grids

template <int T, int P>
void launch_fwd(const LnFwdArgs &a, hipStream_t s)
{
    constexpr int TEAMS = kFwdWaves<T> / T;
    const int64_t wanted = (a.rows + TEAMS - 1) / TEAMS, most = kCus * 32 / kFwdWaves<T>;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(wanted, most)), dim3(kFwdWaves<T> * kWave), 0, s, a);
    };
    if (a.cols % 8 != 0)
        a.res ? go(ln_fwd_kernel<T, P, true, true>) : go(ln_fwd_kernel<T, P, false, true>);
    else
        a.res ? go(ln_fwd_kernel<T, P, true, false>) : go(ln_fwd_kernel<T, P, false, false>);
}

// ---------------------------------------------------------------------------
// Backward.  With xhat = (h - mu) rstd and w = dy gamma of a row:
//   dx = rstd (w - mean(w) - xhat mean(w xhat)) + dres,   dgamma = sum over rows of dy xhat,   dbeta = sum over rows of dy.
// One read of h, dy and dres, one write of dx (6 B an element, 8 with dres).  The column sums stay in registers over the rows that a
// team works on, are added over a workgroup's teams through LDS, and leave the workgroup as one row of partial sums in the
// workspace, which a second launch adds in their order (no atomics: the same bits on every run).  fp32 throughout but for
// h - mu: mu is a double and is subtracted in two parts, since rows whose mean is far above their deviation cancel there.
struct LnBwdArgs {
    const uint16_t *dy, *h, *gamma, *dres;
    const double *stats;
    uint16_t *dx;
    float *partials;  // [groups][2][cols]
    float *sums;      // wide rows: mean(w), mean(w xhat) of each row
    int64_t rows;
    int cols;
};

__device__ __forceinline__ float dpp_sum(float v)
{
    auto add = [](float x, auto ctrl, auto mask) {
        const int o = __builtin_amdgcn_update_dpp(0, (int)f32_to_bits(x), decltype(ctrl)::value, decltype(mask)::value, 0xF, false);
        return x + bits_to_f32((uint32_t)o);
    };
    using std::integral_constant;
    v = add(v, integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});
    v = add(v, integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
    v = add(v, integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
    v = add(v, integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
    v = add(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});
    v = add(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
    return bits_to_f32((uint32_t)__builtin_amdgcn_readlane((int)f32_to_bits(v), 63));
}

__device__ __forceinline__ float element(uint4 v, int k)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    return k & 1 ? bf16hi_to_f32(w[k >> 1]) : bf16lo_to_f32(w[k >> 1]);
}

// SLAB: rows of more pieces than the teams hold; blockIdx.y is the slab of T * P * 64 pieces that this workgroup works on, and a
// launch before has left the two means of each row.
template <int T, int P, int WAVES, bool RES, bool RAGGED, bool SLAB>
__global__ __launch_bounds__(WAVES *kWave) void ln_bwd_kernel(LnBwdArgs a)
{
    constexpr int TEAMS = WAVES / T;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), team = wave / T;
    const int lane = (int)threadIdx.x - team * T * kWave, first = SLAB ? (int)blockIdx.y * T * P * kWave : 0;
    const Row<RAGGED> row(a.cols);
    const float inv_n = 1.0f / (float)a.cols;
    __shared__ float2 red[2][WAVES];
    uint4 gamma[P];
    float dgamma[P][8], dbeta[P][8];
#pragma unroll
    for (int u = 0; u < P; ++u) {
        const int i = first + lane + u * T * kWave;
        // a gain of zero keeps a lane without a piece out of the row's sums (its column sums are not stored)
        gamma[u] = row.load(a.gamma, i);
        if (row.count(i) == 0)
            gamma[u] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            dgamma[u][k] = dbeta[u][k] = 0.0f;
    }
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * TEAMS; r0 < a.rows; r0 += (int64_t)gridDim.x * TEAMS, turn ^= 1) {
        const bool mine = r0 + team < a.rows;
        const int64_t r = mine ? r0 + team : a.rows - 1, at = r * a.cols;
        uint4 h[P], dy[P], dres[RES ? P : 1];
#pragma unroll
        for (int u = 0; u < P; ++u) {
            h[u] = row.load(a.h + at, first + lane + u * T * kWave);
            dy[u] = row.load(a.dy + at, first + lane + u * T * kWave);
            if constexpr (RES)
                dres[u] = row.load(a.dres + at, first + lane + u * T * kWave);
        }
        const double mean = a.stats[2 * r];
        const float mean_hi = (float)mean, mean_lo = (float)(mean - (double)mean_hi), rstd = (float)a.stats[2 * r + 1];
        float c1 = 0.0f, c2 = 0.0f;  // mean(w xhat), mean(w)
        if constexpr (SLAB) {
            c2 = a.sums[2 * r];
            c1 = a.sums[2 * r + 1];
        }
#pragma unroll
        for (int u = 0; u < P; ++u)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float xhat = ((element(h[u], k) - mean_hi) - mean_lo) * rstd, d = element(dy[u], k);
                if constexpr (!SLAB) {
                    const float w = d * element(gamma[u], k);
                    c2 += w;
                    c1 = __builtin_fmaf(w, xhat, c1);
                }
                if (mine) {
                    dgamma[u][k] = __builtin_fmaf(d, xhat, dgamma[u][k]);
                    dbeta[u][k] += d;
                }
            }
        if constexpr (!SLAB) {
            c1 = dpp_sum(c1);
            c2 = dpp_sum(c2);
            if constexpr (T > 1) {
                if ((threadIdx.x & (kWave - 1)) == 0)
                    red[turn][wave] = make_float2(c1, c2);
                __syncthreads();
                c1 = c2 = 0.0f;
#pragma unroll
                for (int w = 0; w < T; ++w) {
                    const float2 v = red[turn][team * T + w];
                    c1 += v.x;
                    c2 += v.y;
                }
            }
            c1 *= inv_n;
            c2 *= inv_n;
        }
        if (!mine)
            continue;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            uint32_t out[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float xhat = ((element(h[u], 2 * k + j) - mean_hi) - mean_lo) * rstd;
                    const float w = element(dy[u], 2 * k + j) * element(gamma[u], 2 * k + j);
                    v[j] = rstd * (w - c2 - xhat * c1);
                    if constexpr (RES)
                        v[j] += element(dres[u], 2 * k + j);
                }
                out[k] = pack_bf16x2(v[0], v[1]);
            }
            row.store(a.dx + at, first + lane + u * T * kWave, make_uint4(out[0], out[1], out[2], out[3]));
        }
    }
    // the teams' column sums, one team after the other
    __shared__ float sums[TEAMS > 1 ? T * P * kWave * 8 : 1];
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        for (int t = 0; TEAMS > 1 && t < TEAMS; ++t) {
            __syncthreads();
            if (team == t)
#pragma unroll
                for (int u = 0; u < P; ++u)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float *at = &sums[(u * 8 + k) * T * kWave + lane];
                        float &v = which ? dbeta[u][k] : dgamma[u][k];
                        if (t > 0)
                            v += *at;
                        *at = v;
                    }
        }
        if (team == TEAMS - 1)
#pragma unroll
            for (int u = 0; u < P; ++u) {
                const int i = first + lane + u * T * kWave, n = row.count(i);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < n)
                        out[(int64_t)which * a.cols + 8 * (int64_t)i + k] = which ? dbeta[u][k] : dgamma[u][k];
            }
    }
}

// mean(w) and mean(w xhat) of wide rows, a workgroup a row
template <bool RAGGED>
__global__ __launch_bounds__(kWideThreads) void ln_bwd_sums_kernel(LnBwdArgs a)
{
    constexpr int T = kWideThreads / kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Row<RAGGED> row(a.cols);
    __shared__ double red[2][T];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const double mean = a.stats[2 * r];
        const float mean_hi = (float)mean, mean_lo = (float)(mean - (double)mean_hi), rstd = (float)a.stats[2 * r + 1];
        float c1 = 0.0f, c2 = 0.0f;
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads) {
            const uint4 h = row.load(a.h + r * a.cols, i), dy = row.load(a.dy + r * a.cols, i), g = row.load(a.gamma, i);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float xhat = ((element(h, k) - mean_hi) - mean_lo) * rstd, w = element(dy, k) * element(g, k);
                c2 += w;
                c1 = __builtin_fmaf(w, xhat, c1);
            }
        }
        const double s2 = team_sum<T>((double)c2, red[0], wave), s1 = team_sum<T>((double)c1, red[1], wave);
        if (threadIdx.x == 0) {
            a.sums[2 * r] = (float)(s2 / (double)a.cols);
            a.sums[2 * r + 1] = (float)(s1 / (double)a.cols);
        }
    }
}

// Adds the workgroups' partial sums in their order: a wave takes 64 columns of one of the two gradients and every 16th row of
// partials, then the 16 waves' sums are added, all in fp64.
constexpr int kColsumWaves = 16;

__global__ __launch_bounds__(kColsumWaves *kWave) void ln_bwd_finish_kernel(const float *__restrict__ partials, int groups, int cols,
                                                                            float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, which = blockIdx.y;
    const int c = (int)blockIdx.x * kWave + lane;
    double s = 0.0;
    if (c < cols)
        for (int g = wave; g < groups; g += kColsumWaves)
            s += (double)partials[((int64_t)g * 2 + which) * cols + c];
    __shared__ double red[kColsumWaves][kWave];
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
#pragma unroll
        for (int w = 1; w < kColsumWaves; ++w)
            s += red[w][lane];
        (which ? dbeta : dgamma)[c] = (float)s;
    }
}

// what a backward call runs on
struct BwdShape {
    int waves_a_row, pieces, waves;  // T, P, WAVES of the kernel
    bool wide;                       // rows longer than T * P * 512 elements
};

BwdShape bwd_shape(int64_t cols)
{
    const int64_t pieces = (cols + 7) / 8;
    if (pieces <= kWave)
        return {1, 1, 8, false};
    if (pieces <= 2 * kWave)
        return {1, 2, 8, false};
    if (pieces <= 4 * kWave)
        return {2, 2, 8, false};
    if (pieces <= 8 * kWave)
        return {4, 2, 8, false};
    return {8, 2, 8, pieces > 16 * kWave};
}

// workgroups, each of which leaves a row of partial sums; of wide rows so many for each slab of columns
int bwd_groups(int64_t rows, int64_t cols, const BwdShape &b)
{
    const int64_t teams = b.waves / b.waves_a_row, slab = (int64_t)b.waves_a_row * b.pieces * kWave * 8;
    const int64_t slabs = b.wide ? (cols + slab - 1) / slab : 1;
    return (int)std::min<int64_t>((rows + teams - 1) / teams, std::max<int64_t>(1, 2 * kCus / slabs));
}

template <int T, int P, int WAVES, bool SLAB = false>
void launch_bwd(const LnBwdArgs &a, int groups, hipStream_t s)
{
    const unsigned slabs = SLAB ? (unsigned)((a.cols + T * P * kWave * 8 - 1) / (T * P * kWave * 8)) : 1u;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups, slabs), dim3(WAVES * kWave), 0, s, a); };
    if (a.cols % 8 != 0)
        a.dres ? go(ln_bwd_kernel<T, P, WAVES, true, true, SLAB>) : go(ln_bwd_kernel<T, P, WAVES, false, true, SLAB>);
    else
        a.dres ? go(ln_bwd_kernel<T, P, WAVES, true, false, SLAB>) : go(ln_bwd_kernel<T, P, WAVES, false, false, SLAB>);
}

}  // namespace

hipError_t launch_layernorm_fwd(const void *x, const void *res, const void *gamma, const void *beta, int64_t rows, int64_t cols,
                                double eps, void *h_out, void *y, double *stats, hipStream_t s)
{
    const LnFwdArgs a{(const uint16_t *)x, (const uint16_t *)res, (const uint16_t *)gamma, (const uint16_t *)beta, (uint16_t *)h_out,
                      (uint16_t *)y, stats, rows, (int)cols, eps};
    const int64_t pieces = (cols + 7) / 8;
    if (pieces <= kWave)
        launch_fwd<1, 1>(a, s);
    else if (pieces <= 2 * kWave)
        launch_fwd<1, 2>(a, s);
    else if (pieces <= 4 * kWave)
        launch_fwd<2, 2>(a, s);
    else if (pieces <= 8 * kWave)
        launch_fwd<4, 2>(a, s);
    else if (pieces <= 16 * kWave)
        launch_fwd<8, 2>(a, s);
    else if (pieces <= 32 * kWave)
        launch_fwd<8, 4>(a, s);
    else {
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(rows, 4 * kCus)), dim3(kWideThreads), 0, s, a);
        };
        if (cols % 8 != 0)
            a.res ? go(ln_fwd_wide_kernel<true, true>) : go(ln_fwd_wide_kernel<false, true>);
        else
            a.res ? go(ln_fwd_wide_kernel<true, false>) : go(ln_fwd_wide_kernel<false, false>);
    }
    return hipGetLastError();
}

size_t layernorm_bwd_bytes(int64_t rows, int64_t cols)
{
    const BwdShape b = bwd_shape(cols);
    return ((size_t)bwd_groups(rows, cols, b) * 2 * (size_t)cols + (b.wide ? 2 * (size_t)rows : 0)) * sizeof(float);
}

hipError_t launch_layernorm_bwd(const void *dy, const void *h, const void *gamma, const double *stats, const void *dres, int64_t rows,
                                int64_t cols, void *dx, float *dgamma, float *dbeta, void *workspace, hipStream_t s)
{
    const BwdShape b = bwd_shape(cols);
    const int groups = bwd_groups(rows, cols, b);
    float *partials = (float *)workspace, *sums = partials + (size_t)groups * 2 * (size_t)cols;
    const LnBwdArgs a{(const uint16_t *)dy, (const uint16_t *)h, (const uint16_t *)gamma, (const uint16_t *)dres, stats,
                      (uint16_t *)dx, partials, sums, rows, (int)cols};
    if (b.wide) {
        const dim3 grid((unsigned)std::min<int64_t>(rows, 4 * kCus));
        if (cols % 8 != 0)
            hipLaunchKernelGGL(ln_bwd_sums_kernel<true>, grid, dim3(kWideThreads), 0, s, a);
        else
            hipLaunchKernelGGL(ln_bwd_sums_kernel<false>, grid, dim3(kWideThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        launch_bwd<8, 2, 8, true>(a, groups, s);
    } else if (b.waves_a_row == 1) {
        b.pieces == 1 ? launch_bwd<1, 1, 8>(a, groups, s) : launch_bwd<1, 2, 8>(a, groups, s);
    } else if (b.waves_a_row == 2) {
        launch_bwd<2, 2, 8>(a, groups, s);
    } else if (b.waves_a_row == 4) {
        launch_bwd<4, 2, 8>(a, groups, s);
    } else {
        launch_bwd<8, 2, 8>(a, groups, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(ln_bwd_finish_kernel, dim3((unsigned)((cols + kWave - 1) / kWave), dbeta != nullptr ? 2 : 1),
                       dim3(kColsumWaves * kWave), 0, s, partials, groups, (int)cols, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace tweo
