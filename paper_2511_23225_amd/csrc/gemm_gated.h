// The gated feed-forward's two products in one tiled kernel (gfx950): a tile of BN rows of B holds BN / 2 rows of the gate and the
// BN / 2 rows of the up projection for the same columns, so that a lane ends up with both values of an element and
// forms act(g) * u where they are.
//
// A 32-row block of B holds, in place 8q + 4b + r, column 8 (q / 2) + 4b + r of 16: the gate's for even q, the up
// projection's for odd.  A lane (l31, lh) of the MFMA layout has places 8q + 4lh + r in its registers 4q + r: gate and up of one
// column are four registers apart.  The rows that a wave brings into LDS, eight at a time, are all of one kind (an even number of
// waves goes round them), so that its base address alone says which.  One row of tokens is bound by the weights (90 MB of INT8: 16 us, 5.7 TB/s),
// 2048 by the matrix instructions between two barriers a stage (11008 columns under 4096, INT8: 200 us, 1.85 POP/s, of 5.4 rounds of tiles; 4096 rows
// 370, 2.0 POP/s).
#pragma once
#include "gemm_common.h"
#include "activation.h"

namespace tweo {

struct GatedDev {
    uint16_t *gu;  // both products as bf16, [M, 2N], or nullptr (FP8)
    GateCoef act;
};

// host side (gemm_gated.hip, gemm_gated_any.hip)
int gated_workgroups(int64_t M, int64_t F, int bm);
hipError_t launch_defer_any_gated(const GemmArgs &a, bool gelu, const GatedDev &gd, hipStream_t s);

// column, of the tile's, of the row-th of the eight rows of B's eight rows number `eight`
__device__ __forceinline__ int gated_column(int eight, int row) { return (eight >> 2) * 16 + ((eight >> 1) & 1) * 8 + row; }

// A wave's part, TM rows by TN / 2 columns: band by band (32 rows) through its own LDS, from where lanes store 8 columns each.
template <typename T, bool INT8, typename ACC>
__device__ __forceinline__ void gated_epilogue(const GemmDev &g, const GatedDev &gd, ACC (&acc)[T::MT][T::NT], uint8_t *smem, int tm,
                                               int tn, int wm, int wn, int lane, int wave, float alpha)
{
    constexpr int COLS = T::TN / 2, PART = COLS * 2, ROW = (INT8 ? 1 : 3) * PART + 16, LPR = COLS / 8, RPP = kWave / LPR;
    static_assert(32 * ROW * (T::THREADS / kWave) <= T::LDS_BYTES, "the bands fit");
    const int l31 = lane & 31, lh = lane >> 5;
    uint8_t *stage = smem + wave * 32 * ROW;
    const int m0 = tm * T::BM + wm * T::TM, n0 = tn * (T::BN / 2) + wn * COLS;
    const int rd_row = lane / LPR, rd_col = n0 + lane % LPR * 8;
    const uint8_t *rd = stage + rd_row * ROW + lane % LPR * 16;
    float gs[INT8 ? T::NT : 1][8], us[INT8 ? T::NT : 1][8];  // INT8: the columns' steps
    if constexpr (INT8) {
#pragma unroll
        for (int j = 0; j < T::NT; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int n = min(n0 + 16 * j + 8 * (k >> 2) + 4 * lh + (k & 3), g.N - 1);
                gs[j][k] = g.cs[(int64_t)n * g.cs_stride];
                us[j][k] = g.cs[((int64_t)g.N + n) * g.cs_stride];
            }
    }
#pragma unroll
    for (int i = 0; i < T::MT; ++i) {
        float rstep = 1.0f;
        if constexpr (INT8)
            rstep = g.rs[(int64_t)min(m0 + 32 * i + l31, g.M - 1) * g.rs_stride];
#pragma unroll
        for (int j = 0; j < T::NT; ++j)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint8_t *to = stage + l31 * ROW + (16 * j + 8 * s + 4 * lh) * 2;
                float h[4];
                if constexpr (INT8) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        h[r] = gated((float)acc[i][j][8 * s + r] * rstep * gs[j][4 * s + r],
                                     (float)acc[i][j][8 * s + 4 + r] * rstep * us[j][4 * s + r], gd.act);
                } else {
                    uint32_t gw[2], uw[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        gw[k] = pack_bf16x2(acc[i][j][8 * s + 2 * k] * alpha, acc[i][j][8 * s + 2 * k + 1] * alpha);
                        uw[k] = pack_bf16x2(acc[i][j][8 * s + 4 + 2 * k] * alpha, acc[i][j][8 * s + 4 + 2 * k + 1] * alpha);
                        h[2 * k] = gated(bf16lo_to_f32(gw[k]), bf16lo_to_f32(uw[k]), gd.act);
                        h[2 * k + 1] = gated(bf16hi_to_f32(gw[k]), bf16hi_to_f32(uw[k]), gd.act);
                    }
                    if (gd.gu != nullptr) {
                        *(uint2 *)(to + PART) = make_uint2(gw[0], gw[1]);
                        *(uint2 *)(to + 2 * PART) = make_uint2(uw[0], uw[1]);
                    }
                }
                if (INT8 && g.out_i8)
                    *(uint32_t *)(stage + l31 * ROW + 16 * j + 8 * s + 4 * lh) =
                        round_to_i8(h[0], g.out_inv_step) | (round_to_i8(h[1], g.out_inv_step) << 8) |
                        (round_to_i8(h[2], g.out_inv_step) << 16) | (round_to_i8(h[3], g.out_inv_step) << 24);
                else
                    *(uint2 *)to = make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
            }
        // the wave reads only what it wrote itself: LDS executes a wave's accesses in order
#pragma unroll
        for (int ps = 0; ps < 32 / RPP; ++ps) {
            const int m = m0 + 32 * i + ps * RPP + rd_row;
            if (m >= g.M || rd_col >= g.N)
                continue;
            const uint8_t *from = rd + ps * RPP * ROW;
            const int64_t at = (int64_t)m * g.N + rd_col;
            if (INT8 && g.out_i8) {
                *(uint2 *)((uint8_t *)g.out + at) = *(const uint2 *)(from - lane % LPR * 8);
                continue;
            }
            *(uint4 *)(g.out + at) = *(const uint4 *)from;
            if (!INT8 && gd.gu != nullptr) {
                uint16_t *gu = gd.gu + 2 * (int64_t)m * g.N + rd_col;
                *(uint4 *)gu = *(const uint4 *)(from + PART);
                *(uint4 *)(gu + g.N) = *(const uint4 *)(from + 2 * PART);
            }
        }
    }
}

}  // namespace tweo
