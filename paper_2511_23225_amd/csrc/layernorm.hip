// LayerNorm to bf16, forward and backward.  Rows of any length; gfx950 only.
// Times in the comments: a call among others in a replayed graph, on three sets of inputs in turn, where no kernel is named alone.
#include <algorithm>
#include <type_traits>
#include "kernels.h"
#include "layernorm.h"

namespace tweo {

namespace {

// ---------------------------------------------------------------------------
// A row is worked on by a team of T waves or, if it is narrow (a norm over the dimensions of a head), of 16 or 8 lanes of a wave
// that has four or eight rows at once (524288x64 forward 140 us with a wave a row, 33; backward 130, 46); lane l of the team
// holds the pieces l, l + 64 T, ... of it, P of them, V elements (4 or 8: 8 or 16 bytes) each, in registers.  RAGGED: cols is no
// multiple of V, so that rows start at any even address and their last piece is short; what they cost is accesses that straddle
// lines (16384x2041 forward 60 us, 2048 wide 45; backward 67 and 51; 4096x4093 37 and 45, 3.0 TB/s).  ONCE: past the caches.

// T = 0 and -1: 16 and 8 lanes
template <int T>
constexpr int kLanes = T < 0 ? 8 : T == 0 ? 16 : T * kWave;

template <int V>
struct Piece {
    uint32_t w[V / 2];  // packed pairs
    __device__ __forceinline__ float at(int k) const { return k & 1 ? bf16hi_to_f32(w[k >> 1]) : bf16lo_to_f32(w[k >> 1]); }
    // keeps the packed form in registers, not its widened values, over what comes next
    __device__ __forceinline__ void keep()
    {
#pragma unroll
        for (int k = 0; k < V / 2; ++k)
            asm volatile("" : "+v"(w[k]));
    }
};

template <int V, bool RAGGED>
struct Row {
    typedef uint32_t vec __attribute__((ext_vector_type(V / 2), aligned(RAGGED ? 2 : 2 * V)));
    int cols, pieces;
    __device__ __forceinline__ explicit Row(int cols_) : cols(cols_), pieces((cols_ + V - 1) / V) {}
    // elements of piece i
    __device__ __forceinline__ int count(int i) const
    {
        const int left = cols - V * i;
        return left < 0 ? 0 : left < V ? left : V;
    }
    // whether one of the team's pieces from i0 on is a ragged row's short one (the same for all lanes)
    template <int T>
    __device__ __forceinline__ bool ends(int i0) const
    {
        return RAGGED && pieces > i0 && pieces <= i0 + kLanes<T>;
    }
    // Piece i, zeros behind a ragged row's end.  Without branches, around which the compiler would wait for one load before it
    // issues the next (4096x4093 backward 60.4 us, now 44.6): a lane without a piece gets the row's last one, and a short piece
    // is taken from the row's last V elements and shifted down. `ending`: the pieces that ends() names.
    template <bool ONCE = false>
    __device__ __forceinline__ Piece<V> load(const uint16_t *p, int i, bool ending) const
    {
        Piece<V> r;
        if (RAGGED && cols < V) {
            const int n = count(i);
            uint32_t e[V];
#pragma unroll
            for (int k = 0; k < V; ++k)
                e[k] = k < n ? p[k] : 0u;
#pragma unroll
            for (int k = 0; k < V / 2; ++k)
                r.w[k] = e[2 * k] | e[2 * k + 1] << 16;
            return r;
        }
        const int last = RAGGED ? cols - V : cols / V * V - V, at = V * i < last ? V * i : last;  // (elements)
        const vec *q = (const vec *)((const uint8_t *)p + (uint64_t)((uint32_t)at * 2u));
        const vec v = ONCE ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
        for (int k = 0; k < V / 2; ++k)
            r.w[k] = v[k];
        if (RAGGED && ending) {
            const int by = i == pieces - 1 ? V * i - at : 0;
            const uint32_t half = by & 1 ? 16 : 0;
#pragma unroll
            for (int k = 0; k < V / 2; ++k)
                r.w[k] = __builtin_amdgcn_alignbit(k + 1 < V / 2 ? r.w[k + 1] : 0u, r.w[k], half);
#pragma unroll
            for (int step = 1; step < V / 2; step *= 2)
#pragma unroll
                for (int k = 0; k < V / 2; ++k)
                    r.w[k] = by & (2 * step) ? (k + step < V / 2 ? r.w[k + step] : 0u) : r.w[k];
        }
        return r;
    }
    template <bool ONCE = false>
    __device__ __forceinline__ void store(uint16_t *p, int i, const Piece<V> &v) const
    {
        vec x;
#pragma unroll
        for (int k = 0; k < V / 2; ++k)
            x[k] = v.w[k];
        const int n = count(i);
        if (RAGGED ? n == V : n > 0) {
            vec *q = (vec *)((uint8_t *)p + (uint64_t)((uint32_t)i * (2u * V)));
            if constexpr (ONCE)
                __builtin_nontemporal_store(x, q);
            else
                *q = x;
        } else if (RAGGED && n > 0) {
#pragma unroll
            for (int k = 0; k < V - 1; ++k)
                if (k < n)
                    p[V * (int64_t)i + k] = (uint16_t)(v.w[k >> 1] >> (16 * (k & 1)));
        }
    }
};

// bytes that a call moves from which on what is not read again soon goes past the caches (the memory-side one has 256 MB)
constexpr int64_t kKeptBytes = 100 << 20;

template <int V>
__device__ __forceinline__ Piece<V> sum_of(const Piece<V> &a, const Piece<V> &b)
{
    // bf16(x + r): the fp32 sum of two bf16 values rounded to bf16 equals the exact sum rounded once
    Piece<V> r;
#pragma unroll
    for (int k = 0; k < V / 2; ++k)
        r.w[k] = pack_bf16x2(a.at(2 * k) + b.at(2 * k), a.at(2 * k + 1) + b.at(2 * k + 1));
    return r;
}

// what stands for a beta that there is not: -0, which leaves a zero the sign that the product gives it
template <int V>
__device__ __forceinline__ Piece<V> nothing_added()
{
    Piece<V> r;
#pragma unroll
    for (int k = 0; k < V / 2; ++k)
        r.w[k] = 0x80008000u;
    return r;
}

template <int V>
__device__ __forceinline__ double sum64(const Piece<V> &v)
{
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < V; ++k)
        s += (double)v.at(k);
    return s;
}

// sum of squared differences of the first n elements
template <int V, bool RAGGED>
__device__ __forceinline__ double squares64(const Piece<V> &v, double mean, int n)
{
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const double d = (double)v.at(k) - mean;
        s += !RAGGED || k < n ? d * d : 0.0;
    }
    return n > 0 ? s : 0.0;
}

// Sum over the lanes of a narrow row's team: its lanes are in one DPP row, and other teams of the wave may have returned.
template <int CTRL>
__device__ __forceinline__ double dpp_add_within(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, false),
                   hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, false);
    return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int CTRL>
__device__ __forceinline__ float dpp_add_within(float v)
{
    return v + bits_to_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f32_to_bits(v), CTRL, 0xF, 0xF, false));
}
// sum over 8 or 16 lanes (a DPP row), in all of them
template <int LANES, typename F>
__device__ __forceinline__ F row_sum(F v)
{
    v = dpp_add_within<0xB1>(v);   // quad_perm: 1 0 3 2
    v = dpp_add_within<0x4E>(v);   // quad_perm: 2 3 0 1
    v = dpp_add_within<0x141>(v);  // row_half_mirror
    return LANES == 8 ? v : dpp_add_within<0x140>(v);  // row_mirror
}

// Sum over the T waves of a team: of each wave through DPP, then through LDS, added in the waves' order by all of them.  `red`: the
// T words of this team for this sum, which are free again two barriers later.
template <int T>
__device__ __forceinline__ double team_sum(double v, double *red, int wave)
{
    if constexpr (T <= 0)
        return row_sum<kLanes<T>>(v);
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

// 1 / sqrt(v), v >= 0, within a few ulp: v_rsq_f64's 2^-24 and one step of third order.  (A square root and a quotient in fp64 are 50
// instructions; with two quotients by the row's length they were a fifth of what a row of 768 issued.)
__device__ __forceinline__ double rsqrt64(double v)
{
    const double y = __builtin_amdgcn_rsq(v), e = __builtin_fma(-v * y, y, 1.0);
    return v > 0.0 && v < __builtin_inf() ? __builtin_fma(y * e, __builtin_fma(e, 0.375, 0.5), y) : y;  // of 0 infinity, of infinity 0; NaN
}

// s / n with 1 / n at hand, rounded once: a row of one value has exactly that value as its mean, and zeros for differences
__device__ __forceinline__ double divided(double s, double n, double inv_n)
{
    const double q = s * inv_n;
    return __builtin_fma(__builtin_fma(-q, n, s), inv_n, q);
}

// ---------------------------------------------------------------------------
// Forward: y = (h - mu) / sqrt(var + eps) * gamma + beta, h = x or bf16(x + residual).  One read of a row (2 B an element, 4 with
// a residual), one write (2, 4): mean and squared differences are taken of the registers, in fp64 as in the pass in front of the
// FP8 cast, whose stored activation has these bits (but where sums in another order and another root, 1e-16 of the value, lie on two
// sides of a rounding boundary).  fp32 in its place: no faster where memory bounds it, 54.4 us and 54.1 at 16384x2048; 19.2 and
// 15.8 at 16384x1024, which the caches hold.  The next row is under way while one is worked on.
// With a residual x and it are read for the last time, and h, the stream, is next read a whole layer later: large calls load and
// store them past the caches (16384x2048 52.4 us, 48.3, the stores alone 53.7; 8192x768, 50 MB, 13.3 and 14.3). 16384x2048 with a
// residual 45.4 us, 5.9 TB/s; 50432x768 51; 8192x768 12.5, where issuing takes half of the time; one row of 2048 6.2, the kernel 2.6.
struct LnFwdArgs {
    const uint16_t *x, *res, *gamma, *beta;
    uint16_t *h, *y;
    double *stats;
    int64_t rows;
    int cols;
    double eps;
};

// (four waves a SIMD: left to itself the compiler takes 130 registers for 16 elements a lane, two more than four waves have;
// 4096x8192 55.0 us -> 49.4)
template <int T, int P, int V, int WAVES, bool RES, bool RAGGED, bool ONCE>
__global__ __launch_bounds__(WAVES *kWave, 4) void ln_fwd_kernel(LnFwdArgs a)
{
    constexpr int TEAMS = WAVES * kWave / kLanes<T>;
    constexpr bool AHEAD = !RAGGED;  // (ragged rows: 16384x2041 80 us with it, 63 without)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), team = T <= 0 ? (int)threadIdx.x / kLanes<T> : wave / std::max(T, 1);
    const int lane = (int)threadIdx.x - team * kLanes<T>;
    const Row<V, RAGGED> row(a.cols);
    const double n = (double)a.cols, inv_n = 1.0 / n;
    __shared__ double red[2][WAVES];
    // a team without a row goes through the last one's sums with the others (barriers) and stores nothing
    Piece<V> nx[P], nr[RES ? P : 1];
    auto request = [&](int64_t r0) {
        const int64_t r = r0 + team < a.rows ? r0 + team : a.rows - 1, at = r * a.cols;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const bool ending = row.template ends<T>(u * kLanes<T>);
            nx[u] = row.template load<ONCE>(a.x + at, lane + u * kLanes<T>, ending);
            if constexpr (RES)
                nr[u] = row.template load<ONCE>(a.res + at, lane + u * kLanes<T>, ending);
        }
    };
    if (AHEAD && (int64_t)blockIdx.x * TEAMS < a.rows)
        request((int64_t)blockIdx.x * TEAMS);
    float gamma[P][V], beta[P][V];
#pragma unroll
    for (int u = 0; u < P; ++u) {
        const int i = lane + u * kLanes<T>;
        const bool ending = row.template ends<T>(u * kLanes<T>);
        const Piece<V> g = row.load(a.gamma, i, ending), b = a.beta != nullptr ? row.load(a.beta, i, ending) : nothing_added<V>();
#pragma unroll
        for (int k = 0; k < V; ++k)
            gamma[u][k] = g.at(k), beta[u][k] = b.at(k);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * TEAMS; r0 < a.rows; r0 += (int64_t)gridDim.x * TEAMS) {
        const bool mine = r0 + team < a.rows;
        const int64_t r = mine ? r0 + team : a.rows - 1, at = r * a.cols;
        if (T <= 1 && !mine)
            return;
        if (!AHEAD)
            request(r0);
        Piece<V> c[P];
#pragma unroll
        for (int u = 0; u < P; ++u) {
            c[u] = nx[u];
            if constexpr (RES)
                c[u] = sum_of(nx[u], nr[u]);
        }
        // before this row's stores: they may overwrite x or the residual, but never another row of them
        if (AHEAD && r0 + (int64_t)gridDim.x * TEAMS < a.rows)
            request(r0 + (int64_t)gridDim.x * TEAMS);
        double s = 0.0;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int i = lane + u * kLanes<T>;
            if (RES && mine)
                row.template store<ONCE>(a.h + at, i, c[u]);
            const double t = sum64(c[u]);
            s += row.count(i) > 0 ? t : 0.0;
        }
        const double mean = divided(team_sum<T>(s, red[0] + team * std::max(T, 0), wave - team * T), n, inv_n);
        double ss = 0.0;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            c[u].keep();
            ss += squares64<V, RAGGED>(c[u], mean, row.count(lane + u * kLanes<T>));
        }
        const double rstd = rsqrt64(__builtin_fma(team_sum<T>(ss, red[1] + team * std::max(T, 0), wave - team * T), inv_n, a.eps));
        if (!mine)
            continue;
        if (a.stats != nullptr && lane == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
#pragma unroll
        for (int u = 0; u < P; ++u) {
            c[u].keep();
            Piece<V> y;
            ln_pairs<V, true>(c[u].w, mean, rstd, gamma[u], beta[u], true, y.w);
            row.store(a.y + at, lane + u * kLanes<T>, y);
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
    const Row<8, RAGGED> row(a.cols);
    const double n = (double)a.cols, inv_n = 1.0 / n;
    __shared__ double red[2][T];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        double s = 0.0;
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads) {
            Piece<8> v = row.load(a.x + r * a.cols, i, true);
            if constexpr (RES) {
                v = sum_of(v, row.load(a.res + r * a.cols, i, true));
                row.store(a.h + r * a.cols, i, v);
            }
            s += sum64(v);
        }
        // h may be x or the residual itself: what this thread has stored is read back, not formed again
        const uint16_t *h = (RES ? a.h : a.x) + r * a.cols;
        const double mean = divided(team_sum<T>(s, red[0], wave), n, inv_n);
        double ss = 0.0;
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads)
            ss += squares64<8, RAGGED>(row.load(h, i, true), mean, row.count(i));
        const double rstd = rsqrt64(__builtin_fma(team_sum<T>(ss, red[1], wave), inv_n, a.eps));
        if (a.stats != nullptr && threadIdx.x == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads) {
            const Piece<8> x = row.load(h, i, true), g = row.load(a.gamma, i, true);
            const Piece<8> b = a.beta != nullptr ? row.load(a.beta, i, true) : nothing_added<8>();
            Piece<8> y;
            float gamma[8], beta[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                gamma[k] = g.at(k), beta[k] = b.at(k);
            ln_pairs<8, true>(x.w, mean, rstd, gamma, beta, true, y.w);
            row.store(a.y + r * a.cols, i, y);
        }
    }
}

constexpr int kCus = 256;  // of an MI355X; a device with more or fewer runs the same grids

template <int T, int P, int V, int WAVES>
void launch_fwd(const LnFwdArgs &a, hipStream_t s)
{
    // as many workgroups as hide each other's barriers: 32 waves a CU, 16 where a team is eight waves and more (4096x8192 52.5
    // us, with 32 54.1 before the stream went past the caches)
    constexpr int TEAMS = WAVES * kWave / kLanes<T>, WAVES_PER_CU = T >= 8 ? 16 : 32;
    const int64_t wanted = (a.rows + TEAMS - 1) / TEAMS, most = kCus * WAVES_PER_CU / WAVES;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(wanted, most)), dim3(WAVES * kWave), 0, s, a);
    };
    if (a.cols % V != 0)
        a.res ? go(ln_fwd_kernel<T, P, V, WAVES, true, true, false>) : go(ln_fwd_kernel<T, P, V, WAVES, false, true, false>);
    else if (a.res && a.rows * a.cols * 8 > kKeptBytes)
        go(ln_fwd_kernel<T, P, V, WAVES, true, false, true>);
    else
        a.res ? go(ln_fwd_kernel<T, P, V, WAVES, true, false, false>) : go(ln_fwd_kernel<T, P, V, WAVES, false, false, false>);
}

// ---------------------------------------------------------------------------
// Backward.  With xhat = (h - mu) rstd and w = dy gamma of a row:
//   dx = rstd (w - mean(w) - xhat mean(w xhat)) + dres,   dgamma = sum over rows of dy xhat,   dbeta = sum over rows of dy.
// One read of h, dy and dres, one write of dx (6 B an element, 8 with dres).  The column sums stay in registers over the rows
// that a team works on, are added over a workgroup's teams through LDS, and leave the workgroup as one row of partial sums in the
// workspace, which a second launch adds in their order (no atomics: the same bits on every run).  512 workgroups of eight waves,
// two a CU: with more of them the partial sums (8 B a column and workgroup) and their addition take what the further waves gain
// (18912x768: 768 of them 37 us in the place of 33).  fp32 throughout but for h - mu: mu is a double and is subtracted in two
// parts, since rows whose mean is far above their deviation cancel there.  (A team adds rows / 256 or fewer rows to one sum; of
// wide rows see below.)  What is read here is read for the last time: large
// calls read past the caches (16384x2048 56.5 us, 51.2; 8192x768, 50 MB, 16.9 and 17.6).  Wide rows on teams of more waves with
// fewer elements each: the sums' registers are what limits the waves. 16384x2048 with dres 51.1 us, 5.3 TB/s (kernels: 45.8 and 4.7
// for the second launch); 18912x768 28.1, 50432x768 59.1, 8192x768 15.9; 257x1001 7.0, the one kernel 6.0.  Rows of more than 8192
// columns read h and dy twice: 2048x16384 87 us, 3.1 TB/s.
struct LnBwdArgs {
    const uint16_t *dy, *h, *gamma, *dres;
    const double *stats;
    uint16_t *dx;
    float *partials;  // [groups][2][cols rounded up to fours]
    float *sums;      // wide rows: mean(w), mean(w xhat) of each row
    int64_t rows;
    int cols;
    // ALONE: workgroups from this one on take the column sums
    int row_groups;
    float *dgamma, *dbeta;
};

// xhat = (h - mu) rstd in fp32.  Where rstd is below 1 both factors are taken by halves and twice, which changes no bit but where h - mu
// itself, of values near bf16's largest, is beyond fp32.
struct Normalizer {
    float scale, mean, rstd, shift;
    __device__ __forceinline__ Normalizer(double mean_d, double rstd_d)
    {
        const float mean_hi = (float)mean_d, r = (float)rstd_d;
        scale = r < 1.0f ? 0.5f : 1.0f;
        mean = mean_hi * scale;
        rstd = r < 1.0f ? 2.0f * r : r;
        shift = (float)(mean_d - (double)mean_hi) * -r;
    }
    __device__ __forceinline__ float operator()(float h) const { return __builtin_fmaf(__builtin_fmaf(h, scale, -mean), rstd, shift); }
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

// Column sums of a call of few rows (ALONE): this workgroup's 64 columns over all rows.  They need the statistics only and not
// the two means of each row, so that other workgroups of the same launch work on dx meanwhile and nothing has to be added
// afterwards; h and dy are read twice, the second time from the caches.  257x768 8.6 us in two launches, 6.0 in one; 512x768 8.7,
// 6.8; 512x4096 15.6, 10.5; 1024x768 9.0, 9.7.
template <int V, int THREADS, bool RAGGED>
__device__ __forceinline__ void column_sums(const LnBwdArgs &a, int group)
{
    constexpr int LANES = 64 / V, PARTS = THREADS / LANES;
    const Row<V, RAGGED> row(a.cols);
    const int lane = threadIdx.x % LANES, part = threadIdx.x / LANES, i = group * LANES + lane;
    float dgamma[V], dbeta[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        dgamma[k] = dbeta[k] = 0.0f;
#pragma unroll 4
    for (int64_t r = part; r < a.rows; r += PARTS) {
        const Piece<V> h = row.load(a.h + r * a.cols, i, true), dy = row.load(a.dy + r * a.cols, i, true);
        const Normalizer normalized(a.stats[2 * r], a.stats[2 * r + 1]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            dgamma[k] = __builtin_fmaf(dy.at(k), normalized(h.at(k)), dgamma[k]);
            dbeta[k] += dy.at(k);
        }
    }
    __shared__ float sums[PARTS][64 + 1];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which) {
            if (a.dbeta == nullptr)
                return;
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < V; ++k)
            sums[part][lane * V + k] = which ? dbeta[k] : dgamma[k];
        __syncthreads();
        const int col = group * 64 + (int)threadIdx.x;
        if (threadIdx.x < 64 && col < a.cols) {
            double s = 0.0;
#pragma unroll 8
            for (int p = 0; p < PARTS; ++p)
                s += (double)sums[p][threadIdx.x];
            (which ? a.dbeta : a.dgamma)[col] = (float)s;
        }
    }
}

// ALONE: the row sums and dx only; column_sums has the rest.  SLAB: rows of more pieces than the teams hold; blockIdx.y is the
// slab of T * P * 64 pieces that this workgroup works on, and a launch before has left the two means of each row.
template <int T, int P, int V, int WAVES, bool RES, bool RAGGED, bool SLAB, bool ONCE, bool ALONE = false>
__global__ __launch_bounds__(WAVES *kWave) void ln_bwd_kernel(LnBwdArgs a)
{
    constexpr int TEAMS = WAVES * kWave / kLanes<T>;
    if constexpr (ALONE)
        if ((int)blockIdx.x >= a.row_groups)
            return column_sums<V, WAVES * kWave, RAGGED>(a, (int)blockIdx.x - a.row_groups);
    const int64_t stride_rows = (int64_t)(ALONE ? a.row_groups : (int)gridDim.x) * TEAMS;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), team = T <= 0 ? (int)threadIdx.x / kLanes<T> : wave / std::max(T, 1);
    const int lane = (int)threadIdx.x - team * kLanes<T>, first = SLAB ? (int)blockIdx.y * P * kLanes<T> : 0;
    const Row<V, RAGGED> row(a.cols);
    const float inv_n = 1.0f / (float)a.cols;
    __shared__ float2 red[2][WAVES];
    float gamma[P][V], dgamma[P][V], dbeta[P][V];
    int turn = 0;
    // the next row under way while one is worked on: where teams are small (16384x1536 47.6 -> 45.6 us; 2048 wide 56.4 -> 59.4) or fill a
    // CU by themselves (4096x8192 61.7 -> 59.3)
    constexpr bool AHEAD = !RAGGED && (T <= 2 || T == 16);
    Piece<V> nh[P], ndy[P], ndres[RES ? P : 1];
    double nmean, nrstd;
    auto request = [&](int64_t r0) {
        const int64_t r = r0 + team < a.rows ? r0 + team : a.rows - 1, at = r * a.cols;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int i = first + lane + u * kLanes<T>;
            const bool ending = row.template ends<T>(first + u * kLanes<T>);
            nh[u] = row.template load<ONCE>(a.h + at, i, ending);
            ndy[u] = row.template load<ONCE>(a.dy + at, i, ending);
            if constexpr (RES)
                ndres[u] = row.template load<ONCE>(a.dres + at, i, ending);
        }
        nmean = a.stats[2 * r], nrstd = a.stats[2 * r + 1];
    };
    if (AHEAD && (int64_t)blockIdx.x * TEAMS < a.rows)
        request((int64_t)blockIdx.x * TEAMS);
#pragma unroll
    for (int u = 0; u < P; ++u) {
        const int i = first + lane + u * kLanes<T>;
        const Piece<V> g = row.load(a.gamma, i, row.template ends<T>(first + u * kLanes<T>));
#pragma unroll
        for (int k = 0; k < V; ++k) {
            gamma[u][k] = g.at(k);
            dgamma[u][k] = dbeta[u][k] = 0.0f;
        }
    }
    // Slabs of wide rows leave few workgroups to a column: the sums of 64 rows are added to others, so that 4096 rows are two sums of
    // 64 terms one after the other.
    constexpr int kHeld = 64;
    float held[2][SLAB ? P : 1][V] = {};
    int rows_held = 0;
    auto hold = [&] {
#pragma unroll
        for (int u = 0; u < (SLAB ? P : 1); ++u)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                held[0][u][k] += dgamma[u][k];
                held[1][u][k] += dbeta[u][k];
                dgamma[u][k] = dbeta[u][k] = 0.0f;
            }
        rows_held = 0;
    };
    for (int64_t r0 = (int64_t)blockIdx.x * TEAMS; r0 < a.rows; r0 += stride_rows, turn ^= 1) {
        const bool mine = r0 + team < a.rows;
        const int64_t r = mine ? r0 + team : a.rows - 1, at = r * a.cols;
        Piece<V> h[P], dy[P], dres[RES ? P : 1];
        if constexpr (!AHEAD)
            request(r0);
#pragma unroll
        for (int u = 0; u < P; ++u) {
            h[u] = nh[u], dy[u] = ndy[u];
            if constexpr (RES)
                dres[u] = ndres[u];
        }
        const Normalizer normalized(nmean, nrstd);
        const float rstd = (float)nrstd;
        if (AHEAD && r0 + stride_rows < a.rows)
            request(r0 + stride_rows);
        float c1 = 0.0f, c2 = 0.0f;  // sums of w xhat, w; then their means
        float xhat[P][V], w[P][V];
#pragma unroll
        for (int u = 0; u < P; ++u) {
            float t1 = 0.0f, t2 = 0.0f;
            const int count = row.count(first + lane + u * kLanes<T>);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                xhat[u][k] = normalized(h[u].at(k));
                // behind a ragged row's end (0 - mean) * rstd may be infinite, and w is 0 there
                if (RAGGED && k > 0)
                    xhat[u][k] = k < count ? xhat[u][k] : 0.0f;
                const float d = dy[u].at(k);
                w[u][k] = d * gamma[u][k];
                if constexpr (!SLAB) {
                    t2 += w[u][k];
                    t1 = __builtin_fmaf(w[u][k], xhat[u][k], t1);
                }
                if (!ALONE && mine) {
                    dgamma[u][k] = __builtin_fmaf(d, xhat[u][k], dgamma[u][k]);
                    dbeta[u][k] += d;
                }
            }
            // (a lane without a piece has another's; its column sums are not stored)
            c1 += count > 0 ? t1 : 0.0f;
            c2 += count > 0 ? t2 : 0.0f;
        }
        if constexpr (SLAB) {
            c2 = a.sums[2 * r];
            c1 = a.sums[2 * r + 1];
        } else {
            c1 = T <= 0 ? row_sum<kLanes<T>>(c1) : dpp_sum(c1);
            c2 = T <= 0 ? row_sum<kLanes<T>>(c2) : dpp_sum(c2);
            if constexpr (T > 1) {
                if ((threadIdx.x & (kWave - 1)) == 0)
                    red[turn][wave] = make_float2(c1, c2);
                __syncthreads();
                c1 = c2 = 0.0f;
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const float2 v = red[turn][team * T + t];
                    c1 += v.x;
                    c2 += v.y;
                }
            }
            c1 *= inv_n;
            c2 *= inv_n;
        }
        if (!mine)
            continue;
        const float k1 = -c1 * rstd, k2 = -c2 * rstd;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            Piece<V> out;
#pragma unroll
            for (int k = 0; k < V / 2; ++k) {
                float v[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    v[j] = __builtin_fmaf(xhat[u][2 * k + j], k1, __builtin_fmaf(w[u][2 * k + j], rstd, k2));
                    if constexpr (RES)
                        v[j] += dres[u].at(2 * k + j);
                }
                out.w[k] = pack_bf16x2(v[0], v[1]);
            }
            row.store(a.dx + at, first + lane + u * kLanes<T>, out);
        }
        if (SLAB && ++rows_held == kHeld)
            hold();
    }
    if constexpr (ALONE)
        return;
    if constexpr (SLAB) {
        hold();
#pragma unroll
        for (int u = 0; u < P; ++u)
#pragma unroll
            for (int k = 0; k < V; ++k)
                dgamma[u][k] = held[0][u][k], dbeta[u][k] = held[1][u][k];
    }
    // the teams' column sums through LDS, then added in the teams' order, four columns a thread
    __shared__ float sums[TEAMS][P * V][kLanes<T>];
    const int stride = (a.cols + 3) & ~3;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * stride;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which)
            __syncthreads();
#pragma unroll
        for (int u = 0; u < P; ++u)
#pragma unroll
            for (int k = 0; k < V; ++k)
                sums[team][u * V + k][lane] = which ? dbeta[u][k] : dgamma[u][k];
        __syncthreads();
        constexpr int QUADS = kLanes<T> * P * V / 4;
#pragma unroll
        for (int q0 = 0; q0 < QUADS; q0 += WAVES * kWave) {
            const int q = q0 + (int)threadIdx.x, l = q % kLanes<T>, part = q / kLanes<T>;
            if (QUADS % (WAVES * kWave) != 0 && q >= QUADS)
                break;
            const int col = V * (first + l + part / (V / 4) * kLanes<T>) + part % (V / 4) * 4;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < TEAMS; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] += sums[t][part * 4 + k][l];
            if (col < a.cols)
                *(float4 *)(out + (int64_t)which * stride + col) = make_float4(v[0], v[1], v[2], v[3]);
        }
    }
}

// mean(w) and mean(w xhat) of wide rows, a workgroup a row: eight elements in fp32, then fp64 (a thread of rows of 2^20 columns adds
// 2048 of them; equal ones in fp32 throughout were off by 2e-5, of 2^22 columns by 7e-5)
template <bool RAGGED>
__global__ __launch_bounds__(kWideThreads) void ln_bwd_sums_kernel(LnBwdArgs a)
{
    constexpr int T = kWideThreads / kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Row<8, RAGGED> row(a.cols);
    __shared__ double red[2][T];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Normalizer normalized(a.stats[2 * r], a.stats[2 * r + 1]);
        double c1 = 0.0, c2 = 0.0;
        for (int i = threadIdx.x; i < row.pieces; i += kWideThreads) {
            const Piece<8> h = row.load(a.h + r * a.cols, i, true), dy = row.load(a.dy + r * a.cols, i, true), g = row.load(a.gamma, i, true);
            const int count = row.count(i);
            float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // (behind a ragged row's end as in ln_bwd_kernel)
                const float xhat = !RAGGED || k < count ? normalized(h.at(k)) : 0.0f, w = dy.at(k) * g.at(k);
                t2 += w;
                t1 = __builtin_fmaf(w, xhat, t1);
            }
            c1 += (double)t1;
            c2 += (double)t2;
        }
        const double s2 = team_sum<T>(c2, red[0], wave), s1 = team_sum<T>(c1, red[1], wave);
        if (threadIdx.x == 0) {
            a.sums[2 * r] = (float)(s2 / (double)a.cols);
            a.sums[2 * r + 1] = (float)(s1 / (double)a.cols);
        }
    }
}

// Adds the workgroups' partial sums: a workgroup takes 4 * kFinLanes columns of one of the two gradients, four a lane, its groups
// of lanes every 128th row of partials, whose sums are then added in their order, all in fp64.  (Lines of 128 B a workgroup, so
// that there are enough workgroups: 512 rows of 768 columns 4.2 us, of 256 B 5.0; a wave 64 columns 10.8.)
constexpr int kFinLanes = 8, kFinThreads = 1024, kFinRows = kFinThreads / kFinLanes;

__global__ __launch_bounds__(kFinThreads) void ln_bwd_finish_kernel(const float *__restrict__ partials, int groups, int cols,
                                                                    float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    const int lane = threadIdx.x % kFinLanes, part = threadIdx.x / kFinLanes, which = blockIdx.y;
    const int stride = (cols + 3) & ~3, c = ((int)blockIdx.x * kFinLanes + lane) * 4;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (c < cols) {
        const float *p = partials + (int64_t)which * stride + c;
#pragma unroll 8
        for (int g = part; g < groups; g += kFinRows) {
            const float4 v = *(const float4 *)(p + (int64_t)g * 2 * stride);
            s[0] += (double)v.x, s[1] += (double)v.y, s[2] += (double)v.z, s[3] += (double)v.w;
        }
    }
    __shared__ double red[kFinRows][kFinLanes * 4 + 1];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        red[part][lane * 4 + k] = s[k];
    __syncthreads();
    const int col = (int)blockIdx.x * kFinLanes * 4 + (int)threadIdx.x;
    if (threadIdx.x < kFinLanes * 4 && col < cols) {
        double t = red[0][threadIdx.x];
        for (int w = 1; w < kFinRows; ++w)
            t += red[w][threadIdx.x];
        (which ? dbeta : dgamma)[col] = (float)t;
    }
}

// few rows, of which a workgroup can take 64 columns as fast as others the rows
bool bwd_alone(int64_t rows, int64_t cols) { return rows <= 512 && cols <= 8192; }

// What a backward call runs on: T, P, V and WAVES of the kernel, lanes with 4 to 12 elements of a row each (their column sums take
// twice as many registers again).  64 lanes for the widths to 256: 16 elements on each of 16 lanes are better on long calls
// (131072x256 42.3 us, 46.6) and worse on others (20000x200 16.2, 13.4; 65536x256 33.5, 32.0).  64 columns on 8 lanes: 65536x64 15.5, on 16 13.7; 524288x64 42.0, 45.9.
struct BwdShape {
    int waves_a_row, pieces, elements, waves;
    bool wide;
};

BwdShape bwd_shape(int64_t cols)
{
    if (cols <= 64)
        return {0, 1, 4, 8, false};
    if (cols <= 128)
        return {0, 1, 8, 8, false};
    if (cols <= 256)
        return {1, 1, 4, 8, false};
    if (cols <= 512)
        return {1, 1, 8, 8, false};
    if (cols <= 768)
        return {1, 3, 4, 8, false};
    if (cols <= 1024)
        return {2, 1, 8, 8, false};
    if (cols <= 1536)
        return {2, 3, 4, 8, false};
    if (cols <= 2048)
        return {4, 1, 8, 8, false};
    if (cols <= 4096)
        return {8, 1, 8, 8, false};
    return {16, 1, 8, 16, cols > 8192};
}

// workgroups, each of which leaves a row of partial sums; of wide rows so many for each slab of columns
int bwd_groups(int64_t rows, int64_t cols, const BwdShape &b)
{
    const int64_t lanes = b.waves_a_row == 0 ? kLanes<0> : b.waves_a_row * kWave,
                   teams = b.waves * kWave / lanes, slab = lanes * b.pieces * b.elements;
    const int64_t slabs = b.wide ? (cols + slab - 1) / slab : 1, most = 16 * kCus / b.waves;
    return (int)std::min<int64_t>((rows + teams - 1) / teams, std::max<int64_t>(1, most / slabs));
}

size_t partial_floats(int64_t cols, int groups) { return (size_t)groups * 2 * (size_t)((cols + 3) / 4 * 4); }

template <int T, int P, int V, int WAVES, bool SLAB = false>
void launch_bwd(const LnBwdArgs &a, int groups, hipStream_t s)
{
    const unsigned slabs = SLAB ? (unsigned)((a.cols + kLanes<T> * P * V - 1) / (kLanes<T> * P * V)) : 1u;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups, slabs), dim3(WAVES * kWave), 0, s, a); };
    if constexpr (!SLAB)
        if (bwd_alone(a.rows, a.cols)) {
            auto alone = [&](int row_groups, int grid) {
                LnBwdArgs b = a;
                b.row_groups = row_groups;
                auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(WAVES * kWave), 0, s, b); };
                if (a.cols % V != 0)
                    a.dres ? run(ln_bwd_kernel<T, P, V, WAVES, true, true, false, false, true>) : run(ln_bwd_kernel<T, P, V, WAVES, false, true, false, false, true>);
                else
                    a.dres ? run(ln_bwd_kernel<T, P, V, WAVES, true, false, false, false, true>) : run(ln_bwd_kernel<T, P, V, WAVES, false, false, false, false, true>);
            };
            const int column_groups = (a.cols + 63) / 64;
            if ((const void *)a.dx != (const void *)a.dy)
                return alone(groups, groups + column_groups);
            alone(0, column_groups);  // in place of dy: the sums first
            return alone(groups, groups);
        }
    if (a.cols % V != 0)
        a.dres ? go(ln_bwd_kernel<T, P, V, WAVES, true, true, SLAB, false>) : go(ln_bwd_kernel<T, P, V, WAVES, false, true, SLAB, false>);
    else if (a.rows * a.cols * (a.dres ? 8 : 6) > kKeptBytes)
        a.dres ? go(ln_bwd_kernel<T, P, V, WAVES, true, false, SLAB, true>) : go(ln_bwd_kernel<T, P, V, WAVES, false, false, SLAB, true>);
    else
        a.dres ? go(ln_bwd_kernel<T, P, V, WAVES, true, false, SLAB, false>) : go(ln_bwd_kernel<T, P, V, WAVES, false, false, SLAB, false>);
}

}  // namespace

hipError_t launch_layernorm_fwd(const void *x, const void *res, const void *gamma, const void *beta, int64_t rows, int64_t cols,
                                double eps, void *h_out, void *y, double *stats, hipStream_t s)
{
    const LnFwdArgs a{(const uint16_t *)x, (const uint16_t *)res, (const uint16_t *)gamma, (const uint16_t *)beta, (uint16_t *)h_out,
                      (uint16_t *)y, stats, rows, (int)cols, eps};
    // the fewest lanes that hold a row with 8 to 16 elements each (131072x256 on 16 lanes 29.9 us, on 64 41.0; two pieces of
    // eight a lane are better than twice the waves: 2048 wide 53.9 us, 59.5).  With a residual two pieces on 16 lanes spill four
    // registers at four waves a SIMD: 131072x256 45.8 us, on 64 lanes 49.6; 65536x256 27.6, 28.2; 400000x256 159, 169, and without
    // spills at three waves 45.5, 25.6, 164.  (Ragged widths of 129 to 255 with a residual: 65536x250 34.6, on 64 lanes 36.6, but
    // 20000x250 14.0, 12.6.)
    if (cols <= 64)
        launch_fwd<-1, 1, 8, 4>(a, s);
    else if (cols <= 128)
        launch_fwd<0, 1, 8, 4>(a, s);
    else if (cols <= 256)
        launch_fwd<0, 2, 8, 4>(a, s);
    else if (cols <= 512)
        launch_fwd<1, 1, 8, 4>(a, s);
    else if (cols <= 768)
        launch_fwd<1, 3, 4, 4>(a, s);
    else if (cols <= 1024)
        launch_fwd<1, 2, 8, 4>(a, s);
    else if (cols <= 1536)
        launch_fwd<2, 3, 4, 4>(a, s);
    else if (cols <= 2048)
        launch_fwd<2, 2, 8, 4>(a, s);
    else if (cols <= 4096)
        launch_fwd<4, 2, 8, 4>(a, s);
    else if (cols <= 8192)
        launch_fwd<8, 2, 8, 8>(a, s);
    else if (cols <= 16384)
        launch_fwd<16, 2, 8, 16>(a, s);
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
    if (bwd_alone(rows, cols))
        return 0;
    const BwdShape b = bwd_shape(cols);
    return (partial_floats(cols, bwd_groups(rows, cols, b)) + (b.wide ? 2 * (size_t)rows : 0)) * sizeof(float);
}

hipError_t launch_layernorm_bwd(const void *dy, const void *h, const void *gamma, const double *stats, const void *dres, int64_t rows,
                                int64_t cols, void *dx, float *dgamma, float *dbeta, void *workspace, hipStream_t s)
{
    const BwdShape b = bwd_shape(cols);
    const int groups = bwd_groups(rows, cols, b);
    float *partials = (float *)workspace, *sums = partials + partial_floats(cols, groups);
    const LnBwdArgs a{(const uint16_t *)dy, (const uint16_t *)h, (const uint16_t *)gamma, (const uint16_t *)dres, stats,
                      (uint16_t *)dx, partials, sums, rows, (int)cols, 0, dgamma, dbeta};
    if (b.wide) {
        const dim3 grid((unsigned)std::min<int64_t>(rows, 4 * kCus));
        if (cols % 8 != 0)
            hipLaunchKernelGGL(ln_bwd_sums_kernel<true>, grid, dim3(kWideThreads), 0, s, a);
        else
            hipLaunchKernelGGL(ln_bwd_sums_kernel<false>, grid, dim3(kWideThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        launch_bwd<16, 1, 8, 16, true>(a, groups, s);
    } else {
        switch (b.waves_a_row * 100 + b.pieces * 10 + b.elements) {
        case 14: launch_bwd<0, 1, 4, 8>(a, groups, s); break;
        case 18: launch_bwd<0, 1, 8, 8>(a, groups, s); break;
        case 114: launch_bwd<1, 1, 4, 8>(a, groups, s); break;
        case 118: launch_bwd<1, 1, 8, 8>(a, groups, s); break;
        case 134: launch_bwd<1, 3, 4, 8>(a, groups, s); break;
        case 218: launch_bwd<2, 1, 8, 8>(a, groups, s); break;
        case 234: launch_bwd<2, 3, 4, 8>(a, groups, s); break;
        case 418: launch_bwd<4, 1, 8, 8>(a, groups, s); break;
        case 818: launch_bwd<8, 1, 8, 8>(a, groups, s); break;
        default: launch_bwd<16, 1, 8, 16>(a, groups, s); break;
        }
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || bwd_alone(rows, cols))
        return e;
    hipLaunchKernelGGL(ln_bwd_finish_kernel, dim3((unsigned)((cols + 4 * kFinLanes - 1) / (4 * kFinLanes)), dbeta != nullptr ? 2 : 1),
                       dim3(kFinThreads), 0, s, partials, groups, (int)cols, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace tweo
