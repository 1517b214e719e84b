// The running sums of query rows, and their tiles of rows as the model has them, for the forms of the attention that work on 16-bit types.
#pragma once

#include "oqm_attend_device.h"

namespace oqm {

// Scores are counted from RAISED below a maximum, and may pass that maximum by SLACK (units of log 2) before sums are scaled anew.  In
// bfloat16 two parts hold a probability to 2^-17 of itself however small it is: it is the maximum itself, and the lag spares most of the
// scaling.  Two parts of binary16 end at 2^-25: counted from the maximum, a probability below 2^-25 would be left out of the values' sums,
// though not out of the sum that divides them.  Counted from 14 below they end at 2^-39, and reach 2^15.9, where binary16 ends at 65504.
// 1000 binary16 tokens over 32 groups, capped / 64 over 128 groups in quant-groups of 32 / 64, us, by RAISED and SLACK: 0 and 8
// 304 / 108.8 / 79.9, 14 and 1.9 306 / 111.2 / 80.5, 15 and 0.9 311 / 112.1 / 82.0, 15 and 0 323 / 113.5 / 85.2.
template <typename T> constexpr float kRaised = __is_same(T, In_f16) ? 14.0f : 0.0f;
template <typename T> constexpr float kSlack = __is_same(T, In_f16) ? 1.9f : 8.0f;

// Caps up to 64 by the plain form of the tanh, larger ones near zero by its series, in kernels of their own (SERIES): 1000 tokens over 32
// groups capped at 30 286 us, at 100 301.  Where one kernel took either, calls without a cap lost by its registers: 3600 groups of 50 along the tokens 42 us
// and 44, 64 tokens over 128 groups in quant-groups of 32 in binary16 110 and 114.
constexpr float kPlainCap = 64.0f * kLog2e;

// The sums of a wave's query rows, and the tiles of rows as the model has them.  A lane's channels of V^T: VU of each of VN runs of
// GS channels.  NZ: sums that are scaled with the others.
template <typename T_, int DP_, int GS_, int MT_, int NZ, bool SERIES>
struct Sums {
    typedef T_ T;
    static constexpr int DP = DP_, GS = GS_, MT = MT_;  // MT: blocks of 16 query rows of a wave
    static constexpr int VU = GS / 16, VN = DP / GS, STEPS = DP / 32;
    static constexpr int PARTS = __is_same(T, In_f16) ? 2 : 1;  // of a query element in bfloat16

    f32x4 o[MT][DP / 16];
    float zero[MT][NZ];
    float ref[MT], sum[MT];  // what the scores and the sums are counted from: RAISED below a maximum that has been; -infinity before there is one

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            ref[m] = -__builtin_inff();
            sum[m] = 0.0f;
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) o[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NZ; ++n) zero[m][n] = 0.0f;
        }
    }
    __device__ __forceinline__ float from(int m) const { return ref[m] == -__builtin_inff() ? 0.0f : ref[m]; }
    // Scores, counted from `base`, to probabilities.  Where a score passes the slack, the tile's are counted from RAISED below the highest
    // of them by their differences.  `ref` is rounded where scores are so large that float32 rounds them (from 2^27 on by 8 and more: 2^8
    // in a probability and beyond what 16 bits hold), so the next tile may count from beside it; it will then pass the slack again.
    __device__ __forceinline__ void probabilities(float (&w)[MT][8], const float (&base)[MT]) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float high = fmaxf(fmaxf(fmaxf(w[m][0], w[m][1]), fmaxf(w[m][2], w[m][3])), fmaxf(fmaxf(w[m][4], w[m][5]), fmaxf(w[m][6], w[m][7])));
            const float level = (ref[m] - base[m]) + kRaised<T>;  // RAISED, or -infinity
            if (__any(high > level + kSlack<T>)) {
                high = fmaxf(high, lane_xor<16>(high));
                high = fmaxf(high, lane_xor<32>(high));
                const float peak = fmaxf(high, level);
                const float by = exp2_of(fminf(kRaised<T> - peak, 0.0f)), down = fmaxf(peak, -__FLT_MAX__);  // sums that have not begun are zero
                ref[m] = base[m] + (peak - kRaised<T>);
                sum[m] *= by;
#pragma unroll
                for (int n = 0; n < DP / 16; ++n) o[m][n] *= by;
#pragma unroll
                for (int n = 0; n < NZ; ++n) zero[m][n] *= by;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[m][i] -= down;
                    if constexpr (kRaised<T> != 0.0f) w[m][i] += kRaised<T>;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[m][i] = exp2_of(w[m][i]);
                sum[m] += w[m][i];
            }
        }
    }
    // Scores are computed from `start` on, and without a cap done; with one they are counted from the maximum as it is put on.
    template <typename ARGS>
    __device__ __forceinline__ void bases(const ARGS& g, float (&base)[MT], float (&start)[MT]) const {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            base[m] = from(m);
            start[m] = g.cap_log2 != 0.0f ? 0.0f : -base[m];
        }
    }
    template <typename ARGS>
    static __device__ __forceinline__ void finish_scores(const ARGS& g, float (&w)[MT][8], const float (&base)[MT]) {
        if constexpr (SERIES) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[m][i] = capped_exactly(w[m][i], g.cap_log2) - base[m];
        } else if (g.cap_log2 != 0.0f) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float high = g.cap_log2 - base[m];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[m][i] = capped(w[m][i], g.cap_log2, high);
            }
        }
    }

    static __device__ __forceinline__ void load_query(const char* p, int quarter, Operand<T> (&q)[STEPS]) {
        asm volatile("" ::: "memory");  // read again for the codes, not kept for them: the registers are wanted
#pragma unroll
        for (int u = 0; u < STEPS; ++u) q[u].w = *reinterpret_cast<const u32x4*>(p + (quarter * (DP / 4) + 8 * u) * 2);
    }
    // 32 tokens of rows as the model has them, from t0; `seen`: of the rows from the first, how many each query row sees.
    __device__ __forceinline__ void rows(const AttendArgs& g, const AttendRows& r, int head, int32_t t0, int32_t tokens, const Operand<T> (&q)[MT][STEPS],
                                         const int32_t (&seen)[MT]) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        const char* k = r.k + head * r.k_head + quarter * (DP / 4) * 2;
        const char* v = r.v + head * r.v_head + a * VU * 2;
        typedef uint32_t Piece __attribute__((ext_vector_type(VU / 2)));
        // what lies behind the last row is read from the last row, and seen by nobody
        u32x4 kx[2][STEPS];
        Piece vx[8][VN];
        auto load_values = [&] {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const char* p = v + (int64_t)min(t0 + 16 * (i / 4) + 4 * quarter + i % 4, tokens - 1) * r.v_row;
#pragma unroll
                for (int n = 0; n < VN; ++n) vx[i][n] = *reinterpret_cast<const Piece*>(p + n * GS * 2);
            }
        };
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char* p = k + (int64_t)min(t0 + 16 * half + a, tokens - 1) * r.k_row;
#pragma unroll
            for (int u = 0; u < STEPS; ++u) kx[half][u] = *reinterpret_cast<const u32x4*>(p + 16 * u);
        }
        if constexpr (MT == 1) load_values();  // in flight with the keys; with two blocks of rows there are no registers for it
        float w[MT][8], base[MT], start[MT];
        bases(g, base, start);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f32x4 d[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) d[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                Operand<T> x;
                x.w = kx[half][u];
#pragma unroll
                for (int m = 0; m < MT; ++m) d[m] = product(x, q[m][u], d[m]);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) w[m][4 * half + i] = __builtin_fmaf(d[m][i], g.scale_log2, start[m]);
        }
        finish_scores(g, w, base);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + 16 * (i / 4) + 4 * quarter + i % 4 >= seen[m]) w[m][i] = -__builtin_inff();
        probabilities(w, base);
        if constexpr (MT > 1) load_values();
        Operand<T> hi[MT], lo[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) split(w[m], hi[m], lo[m]);
#pragma unroll
        for (int n = 0; n < VN; ++n)
#pragma unroll
            for (int u = 0; u < VU; u += 2) {
                Operand<T> even, odd;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = vx[2 * i][n][u / 2], y = vx[2 * i + 1][n][u / 2];
                    even.w[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                    odd.w[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    f32x4 &e = o[m][n * VU + u], &f = o[m][n * VU + u + 1];
                    e = product(even, hi[m], e);
                    e = product(even, lo[m], e);
                    f = product(odd, hi[m], f);
                    f = product(odd, lo[m], f);
                }
            }
    }
};

}  // namespace oqm
