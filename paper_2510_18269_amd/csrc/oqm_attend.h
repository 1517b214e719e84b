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
    f32pair* part_stat;    // [H_q * t_q][splits]: maximum (in units of log 2) and sum
    int64_t q_head, q_row, out_head, out_row;            // bytes
    int32_t k_eff, n_groups, group_tokens, channels, qgroup_log2;
    int32_t t_q, repeat, kv_heads;  // repeat: query heads of a KV head
    int32_t causal, token_axis, bits, meta_bf16;
    uint32_t inv_group_tokens, inv_repeat;
    float scale_log2;      // scale * log2(e); with a cap: scale / softcap
    float cap_log2;        // softcap * log2(e), or 0
    int32_t splits, row_blocks;
};

hipError_t launch_attend(const AttendArgs& a, int dtype, hipStream_t s);

}  // namespace oqm
