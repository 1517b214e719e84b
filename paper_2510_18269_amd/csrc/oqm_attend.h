// What the host side and the kernels of the attention over stored groups share, and the rules that cut its work.
#pragma once

#include <cstring>

#include "oqm_common.h"

namespace oqm {

// Finite, by its bits: the build assumes that arithmetic meets no NaN, so a comparison may not be asked.
inline bool is_number(double x) {
    uint64_t b;
    std::memcpy(&b, &x, sizeof b);
    return (b >> 52 & 0x7ff) != 0x7ff;
}
inline bool is_number(float x) {
    uint32_t b;
    std::memcpy(&b, &x, sizeof b);
    return (b >> 23 & 0xff) != 0xff;
}

struct f32pair {
    float x, y;
};

// No two elements of an output are the same: rows lie inside the steps of the heads, or heads inside the steps of the rows.
inline bool elements_apart(const tom_oqm_view_t& v) {
    if (v.heads < 1 || v.rows < 1) return true;
    const __int128 head_span = (__int128)(v.heads - 1) * v.head_stride + v.channels;  // of one row's heads
    const __int128 row_span = (__int128)(v.rows - 1) * v.row_stride + v.channels;     // of one head's rows
    if (v.rows == 1) return v.heads == 1 || v.head_stride >= v.channels;
    if (v.heads == 1) return v.row_stride >= v.channels;
    return (v.head_stride >= v.channels && v.row_stride >= head_span) || (v.row_stride >= v.channels && v.head_stride >= row_span);
}

// How many recent rows a token of a causal call sees, the last t_q of which are the new tokens' own: none where this is not positive.
// (In this order, since the sum of a token's number and nearly 2^31 rows would pass 32 bits.)
constexpr int32_t recent_seen(int32_t token, int32_t recent_rows, int32_t t_q) { return token + 1 + (recent_rows - t_q); }

struct AttendRows {  // rows as the model has them: in front, or recent
    const char* k;
    const char* v;
    int64_t k_head, k_row, v_head, v_row;  // bytes
    int32_t rows;
};

struct AttendArgs {
    AttendRows front, recent;
    const char* codes[2];  // of the layer, K and V: slot 0, head 0
    const char* meta[2];
    int64_t code_slot, code_head, meta_slot, meta_head;  // bytes
    const int32_t* idx;    // NULL: groups in order
    const char* q;
    char* out;
    float* lse;
    float* part_out;       // [H_q * t_q][splits][d], not normalised; NULL with one split
    f32pair* part_stat;    // [H_q * t_q][splits]: maximum (a score) and sum
    int64_t q_head, q_row, out_head, out_row;            // bytes
    int32_t k_eff, n_groups, group_tokens, channels, qgroup_log2;
    int32_t t_q, repeat, kv_heads;  // repeat: query heads of a KV head
    int32_t causal, token_axis, bits, meta_bf16;
    uint32_t inv_group_tokens, inv_repeat, inv_splits, inv_row_blocks;  // of reciprocal_u32
    // Scores are counted in units of log 2 / score_unit: 1, but in the general form without a cap, which takes the maximum off before it
    // multiplies, so that large scores keep their last bits.
    float scale_log2;      // from dots to scores; with a cap: to the exponent of the tanh, 2 log2(e) scale / softcap
    float cap_log2;        // softcap * log2(e), or 0
    float score_unit;
    int32_t splits, row_blocks;
};

// The kernel a call takes, and how many query rows of a KV head a workgroup of it has (general: a wave).
struct AttendForm {
    bool folded, shared;
    int32_t rows;
};
// Folded: 16-bit rows of 64, 128 or 256 channels, and either quant-groups of 32 channels or more of one token, so that a step of the
// matrix cores (32 channels of keys, 16 of values) lies in one of them, or quant-groups along the tokens, where a tile of 32 tokens
// lies in one of them (mostly empty if they are short, and still the faster: 255 groups of 1 / 5 / 15 tokens, one new token, 135 / 44 /
// 27 us in the general form, 13.4 / 12.9 / 13.1 folded).  Its workgroups have 16 rows, which their waves share, or 16 a wave: 4 heads of
// 128 channels, us of 16 / 64 rows a workgroup, over 64 groups of 196 and over 1024:
//      rows of a head     8           16          17          32          48          64          100
//      64 groups          11.0 / 15.2 11.9 / 15.7 14.6 / 16.4 16.1 / 17.6 17.4 / 19.1 19.2 / 20.8 23.4 / 24.9
//      1024 groups        31.4 / 46.6 32.6 / 47.3 52.8 / 57.5 53.5 / 59.0 76.4 / 72.6 99.1 / 74.9 168 / 131
// so that 17 to 32 rows lose a tenth by the rule, and more of them in short memories.  (32 rows a wave spare a fifth of the instructions but
// leave two waves a SIMD instead of three: 1000 tokens over 32 groups 287 us and 306, 64 over 128 in quant-groups of 32 95 and 105.)
// Shared: other 16-bit forms of the head_dim axis where more than 256 query rows of a head share a tile's reconstruction.  28 query heads on 4,
// quant-groups of 16, us, general / shared:
//      tokens (rows)                   12 (84)     24 (168)    36 (252)    48 (336)    64 (448)
//      64 channels, 64 groups of 50    20.8 / 31.1 26.8 / 33.0 30.2 / 34.8 36.5 / 36.4 41.4 / 37.4
//      128                             33.0 / 38.7 42.2 / 46.5 52.6 / 50.9 60.5 / 53.5 68.3 / 52.2
//      256                             54.7 / 71.2 73.0 / 89.3 87.7 / 87.8 102 / 90.3  118 / 93.1
//      64 channels, 128 groups of 196  56.8 / 48.1 92.5 / 53.8 125 / 58.1  163 / 94.1  212 / 95.0
//      128                             101 / 62.5  172 / 73.7  235 / 79.0  307 / 131   402 / 132
//      256                             173 / 134   289 / 248   399 / 247   519 / 363   676 / 470
// The rule goes by rows alone, where short memories tie.  In long ones the shared form is the faster from 84 rows on, so that they lose up to
// a factor of 3 below 257 rows (with 1 KV head 69 / 53 at 252 rows, with 8 451 / 133).
inline AttendForm attend_form(const tom_oqm_config_t& c, int32_t t_q) {
    const bool tokens = c.qaxis == TOM_QAXIS_TOKENS, f32 = c.out_dtype == TOM_F32;
    const int64_t rows = (int64_t)(c.n_q_heads / c.n_kv_heads) * t_q;
    if (!f32 && (c.head_dim == 64 || c.head_dim == 128 || c.head_dim == 256) && (tokens || c.qgroup >= 32))
        return {true, false, rows <= 16 ? 16 : 64};
    if (!f32 && !tokens && rows > 256) return {false, true, c.head_dim > 128 ? 128 : 256};
    return {false, false, 16};
}

// Waves of the folded kernels that a SIMD holds: what their registers leave, and what the kernels are bound to.  Workgroups have
// one wave on each SIMD, so that it is also the workgroups of a compute unit.  28 query heads on 4, us with one wave less / as it is:
// 256 channels, 1000 tokens over 32 groups of 196 926 / 627, 64 over 128 191 / 133; one more spills: one binary16 token over 2000
// groups of 256 channels 157 (166 with two), over 3600 of 128 channels in quant-groups of 32 126 (179 with three), 64 98 (101).
constexpr int attend_waves(int channels, int qgroup, bool tokens, bool f16, bool few_rows) {
    if (channels == 256) return tokens || (f16 && few_rows) ? 1 : 2;
    if (tokens) return channels == 64 ? 3 : 2;
    if (channels == 64) return 4;
    return (qgroup == 32 && (f16 || few_rows)) || (qgroup == 64 && f16 && few_rows) ? 2 : 3;
}

// Parts that the rows of a call are cut into, each with its own maximum and sum.  Never fewer where there are more rows: the
// workspace of the longest call serves the others.
inline int32_t attend_cuts(const tom_oqm_config_t& c, int32_t t_q, int64_t rows) {
    const AttendForm f = attend_form(c, t_q);
    // Along the tokens' axis a tile of 32 lies in one group, however short.
    if (c.qaxis == TOM_QAXIS_TOKENS) rows = (rows + c.group_tokens - 1) / c.group_tokens * (((int64_t)c.group_tokens + 31) / 32 * 32);
    const int64_t blocks = ((int64_t)(c.n_q_heads / c.n_kv_heads) * t_q + f.rows - 1) / f.rows * c.n_kv_heads;
    int64_t target = 2048, least = 32;  // general: waves, two a SIMD
    if (f.folded) {
        target = 256 * attend_waves(c.head_dim, c.qgroup, c.qaxis == TOM_QAXIS_TOKENS, c.out_dtype == TOM_F16, f.rows == 16);
        least = f.rows == 16 ? 128 : 256;
        if (f.rows > 16) {
            // Rounds of the chip per part, against what they would be if all were full, and what a part of a row costs: written and read
            // again, 1 KB at 5 TB/s, as much as 125 of its tokens.  440 blocks of 7286 rows, us at 1 / 2 / 3 / 4 / 5 / 8 / 9 parts: 394 /
            // 339 / 309 / 283 / 287 / 289 / 373.  (As rows grow the second term falls, so that parts never become fewer.)  From two
            // full rounds up the last one matters little, and the workspace would grow with the call.
            if (blocks >= 2 * target) return 1;
            int64_t best = 1;
            double least_cost = 1e300;
            for (int64_t n = 1; n <= 2 * target / blocks + 2 && n <= (rows + least - 1) / least; ++n) {
                const double rounds = (double)((blocks * n + target - 1) / target) / (double)n * (double)target / (double)blocks;
                const double cost = rounds + 125.0 * (double)n / (double)(rows > 0 ? rows : 1);
                if (cost < least_cost) least_cost = cost, best = n;
            }
            return (int32_t)best;
        }
    } else if (f.shared) {
        target = 256, least = 256;
    }
    int64_t n = target / blocks;
    if (n > (rows + least - 1) / least) n = (rows + least - 1) / least;
    return n < 1 ? 1 : (int32_t)n;
}

// Lanes of the launch of `items` blocks of query rows, each of a part and a KV head.
constexpr uint64_t attend_lanes(const AttendForm& f, uint64_t items) {
    return f.shared ? items * 512 : f.folded ? items * kBlock : (items + kBlock / 64 - 1) / (kBlock / 64) * kBlock;
}

hipError_t launch_attend(const AttendArgs& a, const AttendForm& form, int dtype, hipStream_t s);
void start_attend_shared_bf16(const AttendArgs& g, hipStream_t s);
void start_attend_shared_f16(const AttendArgs& g, hipStream_t s);
void start_attend_bf16_4bit(const AttendArgs& g, const AttendForm& form, hipStream_t s);
void start_attend_bf16_2bit(const AttendArgs& g, const AttendForm& form, hipStream_t s);
void start_attend_f16_4bit(const AttendArgs& g, const AttendForm& form, hipStream_t s);
void start_attend_f16_2bit(const AttendArgs& g, const AttendForm& form, hipStream_t s);

}  // namespace oqm
