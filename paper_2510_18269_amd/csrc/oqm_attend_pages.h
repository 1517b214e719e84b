// What the host side and the kernels of the attention over pages share, and the rules that cut its work.
#pragma once

#include "oqm_pages.h"

namespace oqm {

struct PagesArgs {
    PagePlaces p;
    const char *k, *v;      // of the layer, page 0, head 0
    const char* q;
    char* out;
    const char* prior_out;  // or NULL
    const float* prior_lse;
    float* lse;             // or NULL
    const uint64_t* mask;   // or NULL
    int64_t q_head, q_row, out_head, out_row, prior_head, prior_row;             // bytes
    int64_t lse_head, lse_row, prior_lse_head, prior_lse_row;                    // elements
    int32_t words, causal, channels, kv_heads, repeat;
    uint32_t inv_repeat, inv_kv_heads;
    float scale_log2, cap_log2;  // as in AttendArgs
    // The workgroups of a KV head.  Each sequence's query rows (token by token, the heads of a token beside each other) are cut into blocks,
    // and where `extra` is not zero its rows into parts of one length, the least that the workgroups suffice for.
    uint32_t items, extra;
    int32_t least;               // rows of a part
    int32_t sorted;              // the blocks that see most go first (there are no parts then)
    float* part_out;             // [items][kv_heads][rows of a block][channels], not normalised; written where there are several parts
    f32pair* part_stat;          // [items][kv_heads][rows of a block]: what scores are counted from, and the sum
    uint32_t* unit_first;        // [unit][2]: a block's first item, and its parts
};

// The kernel a call takes: how many query rows of a KV head a workgroup has (16: the few form), and the least that a part of a sequence has.  By the
// average of the sequences, since the host knows no more: all forms take any.
struct PagesForm {
    int32_t block_rows, least;
};
inline PagesForm pages_form(const tom_oqm_pages_t& g, int32_t tokens, int32_t n_q_heads) {
    const int64_t rows = ((int64_t)tokens + g.sequences - 1) / (g.sequences > 0 ? g.sequences : 1) * (n_q_heads / g.heads);
    if (g.dtype == TOM_F32 || rows <= 16) return {16, 128};
    return {rows <= 64 ? 64 : rows <= 1024 || g.channels <= 64 || g.channels > 128 ? 128 : 256, 256};
}

struct PagesCuts {
    uint32_t items, extra;
    uint64_t units;
};
// Blocks of query rows there may be at most, whatever stands in starts, and the further items that let long sequences be cut.
inline PagesCuts pages_cuts(const tom_oqm_pages_t& g, int32_t tokens, int32_t n_q_heads, const PagesForm& f) {
    const uint64_t repeat = (uint64_t)(n_q_heads / g.heads);
    const uint64_t units = g.starts ? (uint64_t)tokens * repeat / f.block_rows + (uint64_t)(g.sequences < tokens ? g.sequences : tokens)
                                    : (uint64_t)tokens * ((repeat + f.block_rows - 1) / f.block_rows);
    const uint64_t target = f.block_rows == 16 ? 1536 : f.block_rows == 256 ? 256 : 512;
    uint64_t extra = target / (uint64_t)g.heads;
    if (extra < 1) extra = 1;
    if (units * (uint64_t)g.heads >= 2 * target || (int64_t)g.table_pages * g.page_rows <= f.least) extra = 0;
    return {(uint32_t)(units + extra), (uint32_t)extra, units};
}

hipError_t launch_attend_pages(const PagesArgs& a, const PagesForm& form, int dtype, hipStream_t s);
void start_attend_pages_f32(const PagesArgs& g, const PagesForm& form, hipStream_t s);
void start_attend_pages_bf16(const PagesArgs& g, const PagesForm& form, hipStream_t s);
void start_attend_pages_f16(const PagesArgs& g, const PagesForm& form, hipStream_t s);

}  // namespace oqm
