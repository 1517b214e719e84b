// Attention over stored groups without reconstructing them: codes enter the matrix products as they are.
//
// With x = code * s + m and (s, m) the same for all channels of a quant-group g of a token t,
//   <q, k_t>      = sum_g s_tg <q, code_t>_g + m_tg sum(q)_g
//   sum_t p_t v_t = sum_t (p_t s_tg) code_t + sum_t p_t m_tg            in the channels of g
// so both products run over the codes, and scales and zeros touch only scores and probabilities, in float32.  A code is exact in
// bfloat16, and cheap: its bits alone are the sub-normal code * 2^-133, which the matrix cores take as such (queries and p * s are
// multiplied by 2^64 against it, so that sums are normal numbers).  An AND gives two operand elements; codes that lie higher in a
// byte come out multiplied by a power of two, which the queries' channels, or the sums at the end, take back.  Queries of binary16
// enter in two bfloat16 parts (exactly), p * s too (2^-17): code * s and m often cancel, so that the rounding of one part would
// show (p * s as one binary16, 2^-12, would spare a seventh of the time).
//
// What this costs in exactness.  The matrix cores align products by the exponents of their operands, and a sub-normal's is that of the
// highest place it could have, so that a product's last places are cut off: measured over 64 tokens, up to 2^-15 of the scale for codes in
// the lowest bits of a byte, 2^-19 for those four bits higher.  With the 2^-17 of p * s (2^-13 of the scale for a code of 15) that is what a value is off by where
// code * s and m cancel; sums over many rows hardly show it (705600 rows: 1.0 % of bfloat16 outputs are rounded to the other side, in plain float32 0.2 %,
// of binary16 7.5 % and 1.3 %; their distance from 64 bits is the same to two digits).  Zeros as quotients by the scales, which the matrix
// cores add up over the same parts of p * s, took 4 to 11 % more time and did not show less.  Along the tokens, where the zeros go with p itself,
// the same costs nothing, and is done: 0.8 % of binary16 outputs over 3600 groups of 50 instead of 2.6 %.
//
// What bounds it, 28 query heads on 4 of 128 channels in groups of 196 tokens, 4 bits.  One new token: memory, 3600 groups (451 MB) in
// 80 us = 5.6 TB/s; few groups, latency: 64 in 7.8 us.  Many tokens: mostly the vector unit, which for every tile takes codes apart and
// multiplies scores and probabilities by scales in every wave: 1000 tokens over 32 groups in quant-groups of 64 with a cap (97 GFLOP) 286
// us, of which it is busy for 213 and the matrix cores for 58, 64 over 128 groups in quant-groups of 32 (23 GFLOP) 96 us, 61 and 14.  For 32
// tokens of 16 rows in quant-groups of 64 a wave issues 24 matrix instructions (384 cycles), 235 of the vector unit (940) and, with a cap, 24
// transcendental ones (384).  About 96 of the 235 take codes apart, alike in the four waves of a workgroup, and 8 a quant-group add the keys' zeros.
// What p * s leaves by one v_dot2 each, instead of a shift and a difference: 301 us against 289.
#pragma once

#include "oqm_attend_sums.h"

namespace oqm {

// What the lanes of a wave wrote to LDS is read by others of it: the wave's LDS operations run in order, so only the compiler must
// keep it.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr float kUp = 0x1p64f, kDown = 0x1p69f;  // 2^64 * 2^-133 = 2^-69

// Operands from packed codes.  In LDS a token's codes are STRIDE bytes from the next one's.
template <int DP, int GS, int BITS>
struct Codes {
    static constexpr int VU = GS / 16, SPG = GS / 32;
    static constexpr int ROW = DP * BITS / 8;  // bytes of a token's codes
    static constexpr int STRIDE = ROW + 16;    // rows spread over the banks
    // Step s of the keys' product in a group: 8 codes of a lane's CQ = GS / 4 channels of it.  `w`: those channels' words.
    static constexpr int CQ = GS / 4, CQ_BYTES = CQ * BITS / 8, CQ_WORDS = CQ_BYTES < 4 ? 1 : CQ_BYTES / 4;
    static __device__ __forceinline__ void key_words(const char* p, uint32_t (&w)[CQ_WORDS]) {
        if constexpr (CQ_BYTES == 2) {
            const uint32_t x = *reinterpret_cast<const uint16_t*>(p);
            w[0] = __builtin_amdgcn_perm(x, x, 0x0c010c00u);  // a byte in each half
        } else if constexpr (CQ_BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (CQ_BYTES == 8) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(p);
            w[0] = x[0];
            w[1] = x[1];
        } else {
            const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = x[i];
        }
    }
    static __device__ __forceinline__ Operand<In_bf16> key_operand(const uint32_t (&w)[CQ_WORDS], int s) {
        Operand<In_bf16> a;
        if constexpr (BITS == 4) {
            const uint32_t x = w[s], y = x >> 8;
            a.w = u32x4{x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u};
        } else {
            const uint32_t x = GS == 32 ? w[0] : s % 2 == 0 ? w[s / 2] : w[s / 2] >> 8;
            a.w = u32x4{x & 0x00030003u, x & 0x000c000cu, x & 0x00300030u, x & 0x00c000c0u};
        }
        return a;
    }
    // The channel of operand element j of step s among the lane's CQ, and what the code is multiplied by there.
    static __device__ __forceinline__ constexpr int key_channel(int s, int j) {
        if (BITS == 4) return 8 * s + j / 2 + 4 * (j % 2);
        if (GS == 32) return j / 2 + 4 * (j % 2);
        return 16 * (s / 2) + 4 * (s % 2) + j / 2 + 8 * (j % 2);
    }
    static __device__ __forceinline__ constexpr float key_factor(int j) {
        return BITS == 4 ? ((j / 2) % 2 ? 16.0f : 1.0f) : j / 2 == 0 ? 1.0f : j / 2 == 1 ? 4.0f : j / 2 == 2 ? 16.0f : 64.0f;
    }
    // Rows of V^T: block n of a group holds channel VU * lane + n of it, for the lane's 8 tokens.
    static __device__ __forceinline__ constexpr float value_factor(int n) {
        return BITS == 4 ? (n % 2 ? 16.0f : 1.0f) : n % 4 == 0 ? 1.0f : n % 4 == 1 ? 4.0f : n % 4 == 2 ? 16.0f : 64.0f;
    }
    static constexpr int VU_BITS = VU * BITS;
    struct ValueWords {
        uint32_t lo[4], hi[4];  // of two tokens each; hi only where a lane's channels of a token fill 32 bits
    };
    static __device__ __forceinline__ void value_words(const char* row0, int a, ValueWords& v) {
        // row0: the group's codes of the lane's first token; its others are 1, 2, 3 and 16 .. 19 rows on
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const char* p = row0 + (i < 2 ? 2 * i : 12 + 2 * i) * STRIDE;
            if constexpr (VU_BITS == 32) {
                const uint32_t x = reinterpret_cast<const uint32_t*>(p)[a], y = reinterpret_cast<const uint32_t*>(p + STRIDE)[a];
                v.lo[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                v.hi[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            } else if constexpr (VU_BITS == 16) {
                const uint32_t x = reinterpret_cast<const uint16_t*>(p)[a], y = reinterpret_cast<const uint16_t*>(p + STRIDE)[a];
                v.lo[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            } else if constexpr (VU_BITS == 8) {
                const uint32_t x = reinterpret_cast<const uint8_t*>(p)[a], y = reinterpret_cast<const uint8_t*>(p + STRIDE)[a];
                v.lo[i] = x | y << 16;
            } else {
                const uint32_t x = reinterpret_cast<const uint8_t*>(p)[a / 2], y = reinterpret_cast<const uint8_t*>(p + STRIDE)[a / 2];
                v.lo[i] = (x | y << 16) >> (4 * (a % 2));
            }
        }
    }
    static __device__ __forceinline__ Operand<In_bf16> value_operand(const ValueWords& v, int n) {
        Operand<In_bf16> r;
        const uint32_t mask = BITS == 4 ? (n % 2 ? 0x00f000f0u : 0x000f000fu) : 0x00030003u << (2 * (n % 4));
        const bool high = BITS == 4 ? n % 4 >= 2 : n >= 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = VU_BITS == 32 && n >= 4 ? v.hi[i] : v.lo[i];
            r.w[i] = (high ? x >> 8 : x) & mask;
        }
        return r;
    }
};

// Quant-groups of GS channels of a token.
template <typename T, int DP, int GS, int BITS, int MT, int NW_, bool SERIES>
struct Folded : Sums<T, DP, GS, MT, DP / GS, SERIES>, Codes<DP, GS, BITS> {
    typedef Sums<T, DP, GS, MT, DP / GS, SERIES> S;
    typedef Codes<DP, GS, BITS> C;
    using S::o, S::zero, S::PARTS, S::STEPS, S::VU;
    using C::ROW, C::STRIDE, C::SPG, C::CQ, C::CQ_BYTES, C::CQ_WORDS;
    static constexpr int NW = NW_;                  // waves that share a staged tile
    static constexpr bool SPREAD = true;
    static constexpr int TT = NW == 1 ? 32 : 64;    // tokens staged
    static constexpr int NG = DP / GS;              // quant-groups of a token
    static constexpr int PIECES = TT * ROW / 16;    // of 16 bytes, of K or of V
    static constexpr int LOADS = (PIECES + NW * 64 - 1) / (NW * 64);
    static constexpr int META = TT * NG * 8;        // bytes of K's or V's pairs in LDS
    static constexpr int STAGE = 2 * TT * STRIDE + 2 * META;
    static constexpr int PLAIN_WAVES = attend_waves(DP, GS, false, __is_same(T, In_f16), NW == 1);
    // a SIMD; the series want registers where there are few left: 256 channels in quant-groups of 32, 64 tokens over 128 groups, capped at 100,
    // with two / one 520 / 342 us (by the plain form, 194)
    static constexpr int WAVES = SERIES && GS <= DP / 4 && PLAIN_WAVES > 1 ? PLAIN_WAVES - 1 : PLAIN_WAVES;

    // ---- staging ----
    struct Fetch {
        u32x4 k[LOADS], v[LOADS];
        uint32_t meta[2 * NG];
        bool seen;        // the token whose pairs the lane holds is one
        uint64_t valid;   // of the tile's tokens
    };
    // The tokens of a tile lie in two groups at most where a group is as long as a tile: their slots are the wave's.
    struct Place {
        int32_t rank, tok, slot0, slot1;
    };
    static __device__ __forceinline__ int32_t slot_at(const AttendArgs& g, int32_t rank) {
        const int32_t at = min(rank, g.k_eff - 1), slot = g.idx ? g.idx[at] : at;
        return rank < g.k_eff && slot >= 0 && slot < g.n_groups ? slot : -1;
    }
    static __device__ __forceinline__ Place place(const AttendArgs& g, int32_t t0) {
        Place p;
        p.rank = (int32_t)div_by((uint32_t)t0, (uint32_t)g.group_tokens, g.inv_group_tokens);
        p.rank = __builtin_amdgcn_readfirstlane(p.rank);
        p.tok = t0 - p.rank * g.group_tokens;
        p.slot0 = p.slot1 = 0;
        if (g.group_tokens >= TT) {
            const int32_t first = slot_at(g, p.rank), second = slot_at(g, p.rank + 1);  // both on their way before one is waited for
            p.slot0 = __builtin_amdgcn_readfirstlane(first);
            p.slot1 = __builtin_amdgcn_readfirstlane(second);
        }
        return p;
    }
    // Slot and row of the tile's token dt; a hole, or what lies behind the last token, is read from slot 0 and not used.
    static __device__ __forceinline__ bool find(const AttendArgs& g, const Place& p, int32_t t0, int32_t tokens, int dt, int32_t& slot, int32_t& tok) {
        if (g.group_tokens >= TT) {
            tok = p.tok + dt;
            slot = p.slot0;
            if (tok >= g.group_tokens) {
                tok -= g.group_tokens;
                slot = p.slot1;
            }
        } else {
            const uint32_t rest = (uint32_t)(p.tok + dt), more = div_by(rest, (uint32_t)g.group_tokens, g.inv_group_tokens);
            tok = (int32_t)(rest - more * (uint32_t)g.group_tokens);
            slot = slot_at(g, p.rank + (int32_t)more);
        }
        const bool is = slot >= 0 && t0 + dt < tokens;
        if (!is) slot = 0;
        return is;
    }
    static __device__ __forceinline__ void fetch(const AttendArgs& g, int head, int32_t tile, Fetch& f) {
        const int32_t t0 = tile * TT, tokens = g.k_eff * g.group_tokens;
        const int tid = NW == 1 ? (int)__lane_id() : (int)threadIdx.x;
        const Place p = place(g, t0);
        const char* kc = g.codes[0] + head * g.code_head;
        const char* vc = g.codes[1] + head * g.code_head;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * NW * 64 + tid;
            int32_t slot, tok;
            find(g, p, t0, tokens, (piece / (ROW / 16)) % TT, slot, tok);
            const int64_t at = slot * g.code_slot + (int64_t)tok * ROW + (piece % (ROW / 16)) * 16;
            f.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kc + at));
            f.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vc + at));
        }
        int32_t slot, tok;
        f.seen = find(g, p, t0, tokens, tid % TT, slot, tok);
        f.valid = __ballot(f.seen);
        if (tid < 2 * TT) {
            const char* m = g.meta[0] + (tid < TT ? 0 : g.meta[1] - g.meta[0]) + head * g.meta_head + slot * g.meta_slot;
            if (g.meta_bf16) {
                const uint32_t* w = reinterpret_cast<const uint32_t*>(m + (int64_t)tok * NG * 4);
#pragma unroll
                for (int i = 0; i < NG; ++i) f.meta[i] = w[i], f.meta[NG + i] = 0;  // all of it on both sides, or it is kept in memory
            } else {
                const u32x2* w = reinterpret_cast<const u32x2*>(m + (int64_t)tok * NG * 8);
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    const u32x2 x = w[i];
                    f.meta[2 * i] = x[0];
                    f.meta[2 * i + 1] = x[1];
                }
            }
        }
    }
    static __device__ __forceinline__ void stage(const AttendArgs& g, const Fetch& f, char* lds) {
        const int tid = NW == 1 ? (int)__lane_id() : (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * NW * 64 + tid;
            if (PIECES % (NW * 64) == 0 || piece < PIECES) {
                char* at = lds + piece / (ROW / 16) * STRIDE + piece % (ROW / 16) * 16;
                *reinterpret_cast<u32x4*>(at) = f.k[i];
                *reinterpret_cast<u32x4*>(at + TT * STRIDE) = f.v[i];
            }
        }
        if (tid < 2 * TT) {
            f32x2* at = reinterpret_cast<f32x2*>(lds + 2 * TT * STRIDE + tid * NG * 8);
            const float unit = tid < TT ? g.scale_log2 * kDown : kUp;  // the scales as the scores, or p * s, want them
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                f32x2 p = {0.f, 0.f};  // a token that is not there must not bring a NaN
                if (f.seen) p = g.meta_bf16 ? widen_pair(f.meta[i]) : f32x2{__uint_as_float(f.meta[2 * i]), __uint_as_float(f.meta[2 * i + 1])};
                p[0] *= unit;
                at[i] = p;
            }
        }
    }

    // Queries, scaled as the codes want them, and the sums of each group's channels in units of the scores.
    struct Query {
        Operand<In_bf16> q[MT][PARTS][STEPS];
        float sum[MT][NG];
    };
    static __device__ __forceinline__ void load(const AttendArgs& g, const char* p, int m, Query& y) {
        const int quarter = (int)__lane_id() >> 4;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            float x[CQ], total = 0.0f;
#pragma unroll
            for (int c = 0; c < CQ; c += 8) load_row<T, 8>(p + (n * GS + quarter * CQ + c) * 2, x + c);
#pragma unroll
            for (int c = 0; c < CQ; ++c) total += x[c];
#pragma unroll
            for (int step = 0; step < SPG; ++step) {
                float z[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = x[C::key_channel(step, j)] * (kUp / C::key_factor(j));
                Operand<In_bf16> hi, lo;
                split(z, hi, lo);
                y.q[m][0][n * SPG + step] = hi;
                if constexpr (PARTS == 2) y.q[m][1][n * SPG + step] = lo;
            }
            total += lane_xor<16>(total);
            total += lane_xor<32>(total);
            y.sum[m][n] = total * g.scale_log2;
        }
    }
    static __device__ __forceinline__ void staged(const AttendArgs&, const char*, const Fetch&, Query&) {}
    static __device__ __forceinline__ int32_t tiles(const AttendArgs& g) { return (g.k_eff * g.group_tokens + TT - 1) / TT; }

    // 32 tokens of a staged tile, from its row `sub`; valid: of the 32.
    __device__ __forceinline__ void stored(const AttendArgs& g, const char* lds, int sub, const Query& y, uint32_t valid) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        const char* kc = lds + sub * STRIDE;
        const char* vc = lds + (TT + sub) * STRIDE;
        const f32x2* km = reinterpret_cast<const f32x2*>(lds + 2 * TT * STRIDE) + sub * NG;
        const f32x2* vm = km + TT * NG;
        float w[MT][8], base[MT], start[MT];
        S::bases(g, base, start);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f32x4 d[MT][NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                uint32_t words[CQ_WORDS];
                C::key_words(kc + (16 * half + a) * STRIDE + i * (GS * BITS / 8) + quarter * CQ_BYTES, words);
#pragma unroll
                for (int m = 0; m < MT; ++m) d[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < SPG; ++s) {
                    const Operand<In_bf16> x = C::key_operand(words, s);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part) d[m][i] = product(x, y.q[m][part][i * SPG + s], d[m][i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2* pair = km + (16 * half + 4 * quarter + i) * NG;
                float x[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) x[m] = start[m];
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    const f32x2 p = pair[n];
#pragma unroll
                    for (int m = 0; m < MT; ++m) x[m] = __builtin_fmaf(p[0], d[m][n][i], __builtin_fmaf(p[1], y.sum[m][n], x[m]));
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) w[m][4 * half + i] = x[m];
            }
        }
        S::finish_scores(g, w, base);
        if (valid != 0xffffffffu) {
            const uint32_t mine = valid >> (4 * quarter);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(mine >> (16 * (i / 4) + i % 4) & 1u))
#pragma unroll
                    for (int m = 0; m < MT; ++m) w[m][i] = -__builtin_inff();
        }
        this->probabilities(w, base);
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            Operand<In_bf16> hi[MT], lo[MT];
            float scaled[MT][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x2 p = vm[(16 * (i / 4) + 4 * quarter + i % 4) * NG + n];
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    scaled[m][i] = w[m][i] * p[0];
                    zero[m][n] = __builtin_fmaf(w[m][i], p[1], zero[m][n]);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) split(scaled[m], hi[m], lo[m]);
            typename C::ValueWords v;
            C::value_words(vc + 4 * quarter * STRIDE + n * (GS * BITS / 8), a, v);
#pragma unroll
            for (int u = 0; u < VU; ++u) {
                const Operand<In_bf16> x = C::value_operand(v, u);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    o[m][n * VU + u] = product(x, hi[m], o[m][n * VU + u]);
                    o[m][n * VU + u] = product(x, lo[m], o[m][n * VU + u]);
                }
            }
        }
    }
    // The sums' units: of the rows (1), or of the codes.
    template <bool TO_CODES>
    __device__ __forceinline__ void rescale() {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) {
                const float f = C::value_factor(n % VU) / kDown;
                o[m][n] *= TO_CODES ? f : 1.0f / f;
            }
    }
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                float z = zero[m][n];
                z += lane_xor<16>(z);
                z += lane_xor<32>(z);
#pragma unroll
                for (int u = 0; u < VU; ++u) o[m][n * VU + u] += z;
            }
    }
};

// Scale and zero of a channel for all tokens of a group:
//   <q, k_t>      = <q s, code_t> + <q, m>            sum_t p_t v_t = s sum_t p_t code_t + m sum_t p_t     over a group's tokens
// so the queries take a group's scales (in three bfloat16 parts), and the sums of a tile, which lies in one group, its values'.
template <typename T, int DP, int BITS, int NW_, bool SERIES>
struct FoldedTokens : Sums<T, DP, (DP < 128 ? DP : 128), 1, 1, SERIES>, Codes<DP, (DP < 128 ? DP : 128), BITS> {
    typedef Sums<T, DP, (DP < 128 ? DP : 128), 1, 1, SERIES> S;
    typedef Codes<DP, (DP < 128 ? DP : 128), BITS> C;
    using S::o, S::STEPS, S::VU, S::VN, S::GS;
    using C::ROW, C::STRIDE, C::SPG, C::CQ, C::CQ_BYTES, C::CQ_WORDS;
    static constexpr int NW = NW_, TT = NW == 1 ? 32 : 64;
    static constexpr bool SPREAD = false;
    static constexpr int PIECES = TT * ROW / 16, LOADS = (PIECES + NW * 64 - 1) / (NW * 64);
    static constexpr int PAIRS = (2 * DP + NW * 64 - 1) / (NW * 64);  // of K and V a lane stages
    static constexpr int STAGE = 2 * TT * STRIDE + 2 * DP * 8;
    static constexpr int WAVES = attend_waves(DP, 0, true, __is_same(T, In_f16), NW == 1);  // a SIMD

    struct Fetch {
        u32x4 k[LOADS], v[LOADS];
        uint32_t meta[2 * PAIRS];
        int32_t rank;
        uint64_t valid;
    };
    static __device__ __forceinline__ int32_t tiles(const AttendArgs& g) { return g.k_eff * ((g.group_tokens + TT - 1) / TT); }
    static __device__ __forceinline__ void fetch(const AttendArgs& g, int head, int32_t tile, Fetch& f) {
        const int tid = NW == 1 ? (int)__lane_id() : (int)threadIdx.x;
        const int32_t parts = (g.group_tokens + TT - 1) / TT;
        f.rank = __builtin_amdgcn_readfirstlane(tile / parts);
        const int32_t tok0 = (tile - f.rank * parts) * TT, tokens = min(TT, g.group_tokens - tok0);
        int32_t slot = g.idx ? g.idx[f.rank] : f.rank;
        slot = __builtin_amdgcn_readfirstlane(slot);
        const bool is = slot >= 0 && slot < g.n_groups;
        f.valid = !is ? 0 : tokens == 64 ? ~uint64_t{0} : (uint64_t{1} << tokens) - 1;
        if (!is) return;  // a hole: its tile is staged as it may be, and not used
        const char* kc = g.codes[0] + head * g.code_head + slot * g.code_slot;
        const int64_t to_v = g.codes[1] - g.codes[0];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * NW * 64 + tid;
            const char* p = kc + (int64_t)(tok0 + min(piece / (ROW / 16) % TT, tokens - 1)) * ROW + piece % (ROW / 16) * 16;
            f.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
            f.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + to_v));
        }
        if (tid * PAIRS < 2 * DP) {
            const bool second = tid * PAIRS >= DP;
            const char* p = g.meta[0] + (second ? g.meta[1] - g.meta[0] : 0) + head * g.meta_head + slot * g.meta_slot;
            const int first = tid * PAIRS - (second ? DP : 0);
            if (g.meta_bf16) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) f.meta[i] = reinterpret_cast<const uint32_t*>(p)[first + i];
            } else {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const u32x2 x = reinterpret_cast<const u32x2*>(p)[first + i];
                    f.meta[2 * i] = x[0];
                    f.meta[2 * i + 1] = x[1];
                }
            }
        }
    }
    static __device__ __forceinline__ void stage(const AttendArgs& g, const Fetch& f, char* lds) {
        const int tid = NW == 1 ? (int)__lane_id() : (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * NW * 64 + tid;
            if (PIECES % (NW * 64) == 0 || piece < PIECES) {
                char* at = lds + piece / (ROW / 16) * STRIDE + piece % (ROW / 16) * 16;
                *reinterpret_cast<u32x4*>(at) = f.k[i];
                *reinterpret_cast<u32x4*>(at + TT * STRIDE) = f.v[i];
            }
        }
        if (tid * PAIRS < 2 * DP) {
            f32x2* at = reinterpret_cast<f32x2*>(lds + 2 * TT * STRIDE) + tid * PAIRS;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                f32x2 p = g.meta_bf16 ? widen_pair(f.meta[i]) : f32x2{__uint_as_float(f.meta[2 * i]), __uint_as_float(f.meta[2 * i + 1])};
                // the values' scales in the units of their sums: what a code is multiplied by depends on its channel
                if (tid * PAIRS >= DP) p[0] *= kDown * value_unit((tid * PAIRS + i) % VU);
                at[i] = p;
            }
        }
    }
    static __device__ __forceinline__ float value_unit(int n) {  // 1 / value_factor, at run time
        return BITS == 4 ? (n % 2 ? 0.0625f : 1.0f) : __uint_as_float((127u - 2u * (uint32_t)(n % 4)) << 23);
    }

    struct Query {
        float x[DP / 4];  // as given, in the order of the operands
        Operand<In_bf16> part[STEPS][3];
        float plain;
        int32_t rank;
    };
    static __device__ __forceinline__ void load(const AttendArgs&, const char* p, int, Query& y) {
        const int quarter = (int)__lane_id() >> 4;
#pragma unroll
        for (int n = 0; n < VN; ++n) {
            float x[CQ];
#pragma unroll
            for (int c = 0; c < CQ; c += 8) load_row<T, 8>(p + (n * GS + quarter * CQ + c) * 2, x + c);
#pragma unroll
            for (int c = 0; c < CQ; ++c) y.x[n * CQ + c] = x[c];
        }
        y.rank = -1;
    }
    // The queries of a group that is another than the last tile's.
    static __device__ __forceinline__ void staged(const AttendArgs& g, const char* lds, const Fetch& f, Query& y) {
        if (f.rank == y.rank) return;
        y.rank = f.rank;
        const int quarter = (int)__lane_id() >> 4;
        const f32x2* pairs = reinterpret_cast<const f32x2*>(lds + 2 * TT * STRIDE);
        float plain = 0.0f;
#pragma unroll
        for (int n = 0; n < VN; ++n) {
            float z[CQ];
#pragma unroll
            for (int c = 0; c < CQ; ++c) {
                const f32x2 p = pairs[n * GS + quarter * CQ + c];
                z[c] = y.x[n * CQ + c] * p[0];
                plain = __builtin_fmaf(y.x[n * CQ + c], p[1], plain);
            }
#pragma unroll
            for (int step = 0; step < SPG; ++step) {
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = z[C::key_channel(step, j)] * (kUp / C::key_factor(j));
                split_key<In_bf16>(w, y.part[n * SPG + step]);
            }
        }
        plain += lane_xor<16>(plain);
        plain += lane_xor<32>(plain);
        y.plain = plain * g.scale_log2;
    }

    __device__ __forceinline__ void stored(const AttendArgs& g, const char* lds, int sub, const Query& y, uint32_t valid) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        const char* kc = lds + sub * STRIDE;
        const char* vc = lds + (TT + sub) * STRIDE;
        const f32x2* vm = reinterpret_cast<const f32x2*>(lds + 2 * TT * STRIDE) + DP;
        float w[1][8], base[1], start[1];
        S::bases(g, base, start);
        const float plain = y.plain + start[0];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < VN; ++i) {
                uint32_t words[CQ_WORDS];
                C::key_words(kc + (16 * half + a) * STRIDE + i * (GS * BITS / 8) + quarter * CQ_BYTES, words);
#pragma unroll
                for (int s = 0; s < SPG; ++s) {
                    const Operand<In_bf16> x = C::key_operand(words, s);
#pragma unroll
                    for (int part = 0; part < 3; ++part) d = product(x, y.part[i * SPG + s][part], d);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) w[0][4 * half + i] = __builtin_fmaf(d[i], g.scale_log2 * kDown, plain);
        }
        S::finish_scores(g, w, base);
        if (valid != 0xffffffffu) {
            const uint32_t mine = valid >> (4 * quarter);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(mine >> (16 * (i / 4) + i % 4) & 1u)) w[0][i] = -__builtin_inff();
        }
        this->probabilities(w, base);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[0][i] *= kUp;
        Operand<In_bf16> hi, lo, ones;
        split(w[0], hi, lo);
        // the zeros go with the sum of the same two parts as the codes: what the parts leave of a probability does not show where
        // the two cancel
        ones.w = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        const float total = product(ones, lo, product(ones, hi, f32x4{0.f, 0.f, 0.f, 0.f}))[0] * (1.0f / kUp);
#pragma unroll
        for (int n = 0; n < VN; ++n) {
            typename C::ValueWords v;
            C::value_words(vc + 4 * quarter * STRIDE + n * (GS * BITS / 8), a, v);
#pragma unroll
            for (int u = 0; u < VU; ++u) {
                const Operand<In_bf16> x = C::value_operand(v, u);
                f32x4 d = product(x, hi, f32x4{0.f, 0.f, 0.f, 0.f});
                d = product(x, lo, d);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 p = vm[n * GS + (4 * quarter + i) * VU + u];
                    o[0][n * VU + u][i] = __builtin_fmaf(d[i], p[0], __builtin_fmaf(total, p[1], o[0][n * VU + u][i]));
                }
            }
        }
    }
    template <bool TO_CODES>
    __device__ __forceinline__ void rescale() {}
    __device__ __forceinline__ void finish() {}
};

// NW == 1: the workgroup's four waves have the same 16 MT query rows, take its tiles in turn, each staging its own, and join at
// the end.  NW == 4: they have 16 MT rows each and share every tile.
template <typename F>
__global__ __launch_bounds__(kBlock, F::WAVES) void attend_folded_kernel(AttendArgs g) {
    typedef typename F::S S;
    typedef typename S::T T;
    constexpr int MT = S::MT, NW = F::NW, TT = F::TT, DP = S::DP, STEPS = S::STEPS, VU = S::VU, VN = S::VN, GS = S::GS;
    constexpr int kStage = NW == 1 ? 4 * F::STAGE : 2 * F::STAGE;
    constexpr int kJoin = NW == 1 ? 4 * (16 * MT * (DP + 4)) * 4 : 0;  // the waves' sums, at the end
    __shared__ __align__(16) char lds[kStage > kJoin ? kStage : kJoin];
    const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
    const Item item = item_of(g, blockIdx.x);
    const uint32_t cut = item.cut;
    const int head = item.head;
    constexpr int kBlockRows = 16 * MT * NW;
    const int32_t rows = g.t_q * g.repeat;
    const int32_t first_row = (int32_t)item.block * kBlockRows, wave_row = first_row + (NW == 1 ? 0 : wave * 16 * MT);

    F f;
    bool there[MT];
    int32_t token[MT], q_head[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int32_t row = wave_row + 16 * m + a;
        there[m] = row < rows;  // one that is not there computes with the first, so that nothing waits for a condition
        token[m] = there[m] ? (int32_t)div_by((uint32_t)row, (uint32_t)g.repeat, g.inv_repeat) : 0;
        q_head[m] = head * g.repeat + (there[m] ? row - token[m] * g.repeat : 0);
    }
    f.clear();
    const bool works = NW == 1 || wave_row < rows;  // a wave of a block's end has no rows but stages with the others
    const int32_t wave_last = (int32_t)div_by((uint32_t)(min(wave_row + 16 * MT, rows) - 1), (uint32_t)g.repeat, g.inv_repeat);
    const Segments s = segments_of(g, min(first_row + kBlockRows, rows) - 1, cut, TT, F::tiles(g));
    // Waves that stage for themselves take every fourth tile, so that the workgroup walks through memory, or, where a run of tiles
    // shares its queries' scales, a run each.
    constexpr int kStep = NW == 1 && F::SPREAD ? 4 : 1;
    int32_t begin = s.begin, end = s.end;
    if constexpr (NW == 1) {
        begin = F::SPREAD ? s.begin + wave : s.begin + (s.end - s.begin) * wave / 4;
        if (!F::SPREAD) end = s.begin + (s.end - s.begin) * (wave + 1) / 4;
    }

    auto from_in = [&](int32_t lo) { return begin >= lo ? begin : begin + (lo - begin + kStep - 1) / kStep * kStep; };
    // Rows in front and recent ones by the same code, so that the sums are held across one copy of it.
    if (works) {
#pragma unroll 1
        for (int segment = 0; segment < 2; ++segment) {
            const AttendRows& r = segment == 0 ? g.front : g.recent;
            const int32_t first = segment == 0 ? 0 : s.front_tiles + s.stored_tiles, tokens = segment == 0 ? g.front.rows : s.recent_rows;
            const int32_t from = from_in(first), to = segment == 0 ? min(end, s.front_tiles) : end;
            if (from >= to) continue;
            const bool causal = segment == 1 && g.causal;
            const int32_t all = causal ? min(tokens, recent_seen(wave_last, g.recent.rows, g.t_q)) : tokens;
            Operand<T> q[MT][STEPS];
            int32_t seen[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                S::load_query(g.q + q_head[m] * g.q_head + token[m] * g.q_row, quarter, q[m]);
                seen[m] = causal ? min(tokens, recent_seen(token[m], g.recent.rows, g.t_q)) : tokens;
            }
            for (int32_t t = from; t < to; t += kStep)
#pragma unroll 1
                for (int sub = 0; sub < TT; sub += 32) {
                    const int32_t t0 = (t - first) * TT + sub;
                    if (t0 < all) f.rows(g, r, head, t0, tokens, q, seen);
                }
        }
    }

    const int32_t stored_end = min(end, s.front_tiles + s.stored_tiles);
    if (from_in(s.front_tiles) < stored_end) {
        char* const mine = lds + (NW == 1 ? wave * F::STAGE : 0);
        typename F::Fetch next;
        int32_t t = from_in(s.front_tiles);
        F::fetch(g, head, t - s.front_tiles, next);  // the first tile is on its way while the queries are read
        typename F::Query query;
#pragma unroll
        for (int m = 0; m < MT; ++m) F::load(g, g.q + q_head[m] * g.q_head + token[m] * g.q_row, m, query);
        f.template rescale<true>();
        for (int buffer = 0; t < stored_end; t += kStep, buffer ^= 1) {
            char* const here = mine + (NW == 1 ? 0 : buffer * F::STAGE);
            const uint64_t valid = next.valid;
            F::stage(g, next, here);
            if constexpr (NW == 1) wave_sync();
            else __syncthreads();  // the other buffer is written only behind the next of these, when all have read it
            if (works && valid) F::staged(g, here, next, query);
            if (t + kStep < stored_end) F::fetch(g, head, t + kStep - s.front_tiles, next);
            if (works) {
#pragma unroll 1
                for (int sub = 0; sub < TT; sub += 32)
                    if ((uint32_t)(valid >> sub)) f.stored(g, here, sub, query, (uint32_t)(valid >> sub));
            }
            if constexpr (NW == 1) wave_sync();
        }
        f.template rescale<false>();
    }

#pragma unroll
    for (int m = 0; m < MT; ++m) {
        f.sum[m] += lane_xor<16>(f.sum[m]);
        f.sum[m] += lane_xor<32>(f.sum[m]);
    }
    f.finish();

    typedef typename Element<T>::type E;
    if constexpr (NW == 1) {
        // the waves' sums by LDS: [wave][row][DP + 4], the row's maximum and sum behind it
        constexpr int kRow = DP + 4;
        float* const mine = reinterpret_cast<float*>(lds) + wave * 16 * MT * kRow;
        __syncthreads();  // staged tiles have been read
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float* const row = mine + (16 * m + a) * kRow;
#pragma unroll
            for (int n = 0; n < VN; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int u = 0; u < VU; u += 2)
                        *reinterpret_cast<f32x2*>(row + n * GS + (4 * quarter + i) * VU + u) = f32x2{f.o[m][n * VU + u][i], f.o[m][n * VU + u + 1][i]};
            if (quarter == 0) *reinterpret_cast<f32x2*>(row + DP) = f32x2{f.ref[m], f.sum[m]};
        }
        __syncthreads();
        constexpr int kLanes = DP / 4;  // of a row
        const float* const base = reinterpret_cast<const float*>(lds);
        for (int r = (int)threadIdx.x / kLanes; r < min(16 * MT, rows - first_row); r += kBlock / kLanes) {
            const int c = (int)threadIdx.x % kLanes * 4;
            f32x2 stat[4];
            float high = -__builtin_inff(), total = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                stat[w] = *reinterpret_cast<const f32x2*>(base + (w * 16 * MT + r) * kRow + DP);
                high = fmaxf(high, stat[w][0]);
            }
            const float from = high == -__builtin_inff() ? 0.0f : high;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float by = exp2_of(stat[w][0] - from);
                total = __builtin_fmaf(by, stat[w][1], total);
                x += *reinterpret_cast<const f32x4*>(base + (w * 16 * MT + r) * kRow + c) * by;
            }
            const int32_t tok = (int32_t)div_by((uint32_t)(first_row + r), (uint32_t)g.repeat, g.inv_repeat);
            const int32_t qh = head * g.repeat + first_row + r - tok * g.repeat;
            const int64_t at = (int64_t)qh * g.t_q + tok;
            if (g.splits > 1) {
                *reinterpret_cast<f32x4*>(g.part_out + (at * g.splits + cut) * DP + c) = x;
                if (c == 0) g.part_stat[at * g.splits + cut] = f32pair{high, total};
            } else {
                const float by = total > 0.0f ? 1.0f / total : 0.0f;
                typedef E Vec __attribute__((ext_vector_type(4)));
                Vec y;
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = (E)(x[i] * by);
                *reinterpret_cast<Vec*>(g.out + qh * g.out_head + tok * g.out_row + (int64_t)c * 2) = y;
                if (c == 0 && g.lse) g.lse[at] = total > 0.0f ? (high + __builtin_amdgcn_logf(total)) * kLn2 : -__builtin_inff();
            }
        }
    } else {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (!there[m]) continue;
            const int64_t at = (int64_t)q_head[m] * g.t_q + token[m];
            const float by = f.sum[m] > 0.0f ? 1.0f / f.sum[m] : 0.0f;
#pragma unroll
            for (int n = 0; n < VN; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = n * GS + (4 * quarter + i) * VU;
                    if (g.splits > 1) {
                        typedef float Vec __attribute__((ext_vector_type(VU)));
                        Vec y;
#pragma unroll
                        for (int u = 0; u < VU; ++u) y[u] = f.o[m][n * VU + u][i];
                        *reinterpret_cast<Vec*>(g.part_out + (at * g.splits + cut) * DP + c) = y;
                    } else {
                        typedef E Vec __attribute__((ext_vector_type(VU)));
                        Vec y;
#pragma unroll
                        for (int u = 0; u < VU; ++u) y[u] = (E)(f.o[m][n * VU + u][i] * by);
                        *reinterpret_cast<Vec*>(g.out + q_head[m] * g.out_head + token[m] * g.out_row + (int64_t)c * 2) = y;
                    }
                }
            if (quarter == 0) {
                if (g.splits > 1) g.part_stat[at * g.splits + cut] = f32pair{f.ref[m], f.sum[m]};
                else if (g.lse) g.lse[at] = f.sum[m] > 0.0f ? (f.ref[m] + __builtin_amdgcn_logf(f.sum[m])) * kLn2 : -__builtin_inff();
            }
        }
    }
}

template <typename F16, typename F64>  // of 16 and of 64 rows a workgroup
void start_folded_form(const AttendArgs& g, const AttendForm& form, hipStream_t s) {
    const dim3 grid((uint32_t)((int64_t)g.row_blocks * g.splits * g.kv_heads)), block(kBlock);
    if (form.rows == 16) launch(attend_folded_kernel<F16>, grid, block, 0, s, g);
    else launch(attend_folded_kernel<F64>, grid, block, 0, s, g);
}

template <typename T, int DP, int GS, int BITS>
void start_folded(const AttendArgs& g, const AttendForm& form, hipStream_t s) {
    if (g.cap_log2 > kPlainCap) start_folded_form<Folded<T, DP, GS, BITS, 1, 1, true>, Folded<T, DP, GS, BITS, 1, 4, true>>(g, form, s);
    else start_folded_form<Folded<T, DP, GS, BITS, 1, 1, false>, Folded<T, DP, GS, BITS, 1, 4, false>>(g, form, s);
}

template <typename T, int DP, int BITS>
void start_folded_tokens(const AttendArgs& g, const AttendForm& form, hipStream_t s) {
    if (g.cap_log2 > kPlainCap) start_folded_form<FoldedTokens<T, DP, BITS, 1, true>, FoldedTokens<T, DP, BITS, 4, true>>(g, form, s);
    else start_folded_form<FoldedTokens<T, DP, BITS, 1, false>, FoldedTokens<T, DP, BITS, 4, false>>(g, form, s);
}

template <typename T, int BITS>
void start_folded_of(const AttendArgs& g, const AttendForm& form, hipStream_t s) {
    if (g.token_axis) {
        if (g.channels == 64) start_folded_tokens<T, 64, BITS>(g, form, s);
        else if (g.channels == 128) start_folded_tokens<T, 128, BITS>(g, form, s);
        else start_folded_tokens<T, 256, BITS>(g, form, s);
        return;
    }
    const int gs = 1 << g.qgroup_log2;
    if (g.channels == 64) {
        if (gs == 32) start_folded<T, 64, 32, BITS>(g, form, s);
        else start_folded<T, 64, 64, BITS>(g, form, s);
    } else if (g.channels == 128) {
        if (gs == 32) start_folded<T, 128, 32, BITS>(g, form, s);
        else if (gs == 64) start_folded<T, 128, 64, BITS>(g, form, s);
        else start_folded<T, 128, 128, BITS>(g, form, s);
    } else {
        if (gs == 32) start_folded<T, 256, 32, BITS>(g, form, s);
        else if (gs == 64) start_folded<T, 256, 64, BITS>(g, form, s);
        else start_folded<T, 256, 128, BITS>(g, form, s);
    }
}

}  // namespace oqm
