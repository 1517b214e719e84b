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
    int32_t by_terms;            // the powers of scale_log2 that the tanh's first terms want are float32 numbers
    // The workgroups of a KV head.  Each sequence's query rows (token by token, the heads of a token beside each other) are cut into blocks,
    // and where `extra` is not zero its rows into parts of one length, the least that the workgroups suffice for.
    uint32_t items, extra;
    int32_t least;               // rows of a part
    int32_t sorted;              // the blocks that see most go first (there are no parts then)
    float* part_out;             // [items][kv_heads][rows of a block][channels], not normalised; written where there are several parts
    f32pair* part_stat;          // [items][kv_heads][rows of a block]: what scores are counted from, and the sum
    uint32_t* unit_first;        // [unit][2]: a block's first item, and its parts
};

// The kernel a call takes: how many query rows of a KV head a workgroup has (16: the few form), whether two waves share them and halve what they see (SPLIT),
// and how a sequence's rows are cut into parts: `least` rows each, `target` workgroups in all.  By the average of the sequences, since the host knows no more: all
// forms take any.
struct PagesForm {
    int32_t block_rows, least, target;
    bool split;
};
// Blocks of query rows there may be at most, whatever stands in starts.
inline uint64_t pages_units(const tom_oqm_pages_t& g, int32_t tokens, int32_t n_q_heads, int32_t block_rows) {
    const uint64_t repeat = (uint64_t)(n_q_heads / g.heads);
    return g.starts ? (uint64_t)tokens * repeat / block_rows + (uint64_t)(g.sequences < tokens ? g.sequences : tokens)
                    : (uint64_t)tokens * ((repeat + block_rows - 1) / block_rows);
}
// 28 query heads on 4 of 128 channels in bfloat16, us of one form / the next:
//      16 / 64 rows:   16 sequences of 1000 to 9000 rows, 4 tokens (28 query rows) 63.2 / 43.7; 13 tokens (91) 21.1 by 64 and by 128
//      64 / 128:       the same sequences, 8 tokens (56 query rows) 39.5 / 51.8
//      128 / 256:      4 sequences of 2000 to 7900 rows, 43 to 52 tokens (301 to 364) 39.4 / 50.9; 3 prompts of 1467 to 1994 tokens 386 / 371, one of 8192 532 / 483, but of 64
//                      channels 216 / 255.  Of 256 channels 256 rows would leave half the registers.
//      128, SPLIT:     43 to 52 tokens 41.5 / 37.6: half as many parts to write and join
// All of these are batches whose sequences are alike.  One form for all of a call costs those that are not: 63 tokens over 1000 to 30000 rows 435 us, a prompt of 4000 tokens 187, in one call
// 994 (256 rows a workgroup, of which a token has 7); in a call each they take the sum.
// Workgroups, us: few form, 512 / 768 / 1024 / 1536: 48 sequences of 40 to 30000 rows, a token each, 355 / 296 / 299 / 290, one of 705 K rows 259 / 297 / 265 / 271, 256 of 40 to 1000
// rows 51 / 61 / 61 / 63, 64 channels 349 / 374 / 354 / 335, 256 channels 355 / 336 / 324 / 320.  64 rows, 512 / 640 / 768: 16 sequences, 8 tokens 49.9 / 48.2 / 48.3, 4 tokens 38.1 / 37.5 /
// 39.5.
inline PagesForm pages_form(const tom_oqm_pages_t& g, int32_t tokens, int32_t n_q_heads) {
    const int64_t rows = (int64_t)tokens * (n_q_heads / g.heads);
    auto on_average = [&](int64_t most) { return rows <= most * g.sequences; };  // not rounded: a token more in a batch must not move all of it to fewer bits
    if (g.dtype == TOM_F32 || on_average(16)) return {16, 128, 1536, false};
    if (on_average(64)) return {64, 256, 640, false};
    if (!on_average(1024) && g.channels > 64 && g.channels <= 128) return {256, 256, 256, false};
    if (g.channels <= 128 && pages_units(g, tokens, n_q_heads, 128) * (uint64_t)g.heads < 512) return {128, 256, 256, true};
    return {128, 256, 512, false};
}

// Sequences among whose blocks every workgroup looks for those that see most; of more, each finds its own alone.  Tokens of sequences of up to 600 (8192: 100) rows, looked for
// among all / found alone / with one token each, where there is nothing to find, us: 1024 sequences 239 / 140 / 134, 2048 965 / 266 / 257, 8192 10894 / 367 / 283.
constexpr int32_t kMostSorted = 512;

struct PagesCuts {
    uint32_t items, extra;
    uint64_t units;
};
// Items of a KV head: its blocks, and further ones that let long sequences be cut where the blocks do not fill the chip.  Where they do, by their number, nothing is cut, and a
// sequence far longer than the others is read by one workgroup a KV head alone: 799 tokens over 40 to 600 rows each 120 us, with an 800th over 30000 rows 798, over 700 K rows 16.9 ms
// (alone, cut over the chip, 260 us).  Such a sequence is better given a call of its own.
inline PagesCuts pages_cuts(const tom_oqm_pages_t& g, int32_t tokens, int32_t n_q_heads, const PagesForm& f) {
    const uint64_t units = pages_units(g, tokens, n_q_heads, f.block_rows);
    const uint64_t most = (uint64_t)f.target / (uint64_t)g.heads;
    uint64_t extra = most;
    // Blocks of many rows: no more than run at a time, one round of the chip.  (The 264 workgroups of 4 sequences on 256 compute units took 50.8 us, 216 37.6.)
    if (f.block_rows > 64) extra = most > units + most / 4 ? most - units : most / 4;
    if (extra < 1) extra = 1;
    if (units * (uint64_t)g.heads >= 2 * (uint64_t)f.target || (int64_t)g.table_pages * g.page_rows <= f.least) extra = 0;
    return {(uint32_t)(units + extra), (uint32_t)extra, units};
}

hipError_t launch_attend_pages(const PagesArgs& a, const PagesForm& form, int dtype, hipStream_t s);
void start_attend_pages_f32(const PagesArgs& g, const PagesForm& form, hipStream_t s);
void start_attend_pages_bf16(const PagesArgs& g, const PagesForm& form, hipStream_t s);
void start_attend_pages_f16(const PagesArgs& g, const PagesForm& form, hipStream_t s);

}  // namespace oqm
