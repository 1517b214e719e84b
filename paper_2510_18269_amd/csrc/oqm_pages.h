// Rows of several sequences in pages: what the host side checks, and how a kernel finds a row.
#pragma once

#include "oqm_attend.h"
#include "oqm_common.h"
#include "oqm_device.h"

namespace oqm {

constexpr int32_t kMaxSequences = 1 << 20;
constexpr int64_t kMaxPagedRows = 0x7fffffff - 4096;  // a tile's last row stays inside 32 bits

// The pages of a layer as a kernel addresses them.  A row's place is counted in 16 bytes from the head's first page, in 32 bits.
struct PagePlaces {
    const int32_t* table;
    const int32_t* rows;
    const int32_t* starts;  // NULL: one token each
    uint32_t page_step, row_step;  // 16 bytes
    int64_t head_bytes;
    int32_t sequences, table_pages, n_pages, page_rows;
    uint32_t inv_page_rows;
    int32_t capacity;       // rows that a table has entries for
    int32_t tokens;         // of the call
};

inline int bytes_of_dtype(int32_t dtype) { return dtype == TOM_F32 ? 4 : 2; }

// Checks everything but the layer, and fills in all of `p` but the tokens.
inline tom_status_t check_pages(const tom_oqm_pages_t* g, PagePlaces& p) {
    constexpr int64_t kMaxStride = int64_t{1} << 40;  // elements; far beyond any device tensor
    if (!g) return fail(TOM_ERR_INVALID_ARG, "pages is NULL");
    if (g->dtype != TOM_F32 && g->dtype != TOM_BF16 && g->dtype != TOM_F16) return fail(TOM_ERR_INVALID_ARG, "the dtype of the pages is not a tom_dtype_t");
    if (g->channels < 8 || g->channels > 256 || g->channels % 8) return fail(TOM_ERR_INVALID_ARG, "channels = %d of the pages must be a multiple of 8 in [8, 256]", g->channels);
    if (g->n_layers < 1 || g->n_pages < 1 || g->heads < 1 || g->page_rows < 1)
        return fail(TOM_ERR_INVALID_ARG, "the pages need a layer, a page, a head and a row at least");
    if (g->sequences < 0 || g->table_pages < 0) return fail(TOM_ERR_INVALID_ARG, "sequences or table_pages is negative");
    if (g->sequences > kMaxSequences) return fail(TOM_ERR_UNSUPPORTED, "%d sequences: at most %d per call", g->sequences, kMaxSequences);
    if ((int64_t)g->table_pages * g->page_rows > kMaxPagedRows)
        return fail(TOM_ERR_UNSUPPORTED, "%d pages of %d rows: at most %lld rows per sequence", g->table_pages, g->page_rows, (long long)kMaxPagedRows);
    const int e = bytes_of_dtype(g->dtype);
    const int64_t strides[4] = {g->layer_stride, g->page_stride, g->head_stride, g->row_stride};
    const int32_t sizes[4] = {g->n_layers, g->n_pages, g->heads, g->page_rows};
    int64_t bytes[4];
    int order[4] = {0, 1, 2, 3};
    for (int i = 0; i < 4; ++i) {
        if (strides[i] < 0 || strides[i] > kMaxStride) return fail(TOM_ERR_INVALID_ARG, "strides of the pages must be in [0, 2^40] elements");
        bytes[i] = sizes[i] > 1 ? strides[i] * e : 0;  // the stride of a size of one says nothing
        if (bytes[i] & 15) return fail(TOM_ERR_INVALID_ARG, "strides of the pages must be multiples of 16 bytes");
    }
    // no two elements are the same: by growing stride, each steps over all that lies inside it
    for (int i = 1; i < 4; ++i)
        for (int j = i; j > 0 && bytes[order[j]] < bytes[order[j - 1]]; --j) {
            const int t = order[j];
            order[j] = order[j - 1];
            order[j - 1] = t;
        }
    __int128 span = (__int128)g->channels * e;
    for (int i = 0; i < 4; ++i) {
        if (sizes[order[i]] == 1) continue;
        if (bytes[order[i]] < span) return fail(TOM_ERR_INVALID_ARG, "layers, pages, heads or rows of the pages overlap");
        span += (__int128)(sizes[order[i]] - 1) * bytes[order[i]];
    }
    if ((__int128)(g->n_pages - 1) * bytes[1] + (__int128)(g->page_rows - 1) * bytes[3] + 1024 >= (__int128)1 << 36)
        return fail(TOM_ERR_UNSUPPORTED, "a layer's pages span 2^36 bytes and more");
    if (g->sequences > 0) {
        if (!g->k || !g->v) return fail(TOM_ERR_INVALID_ARG, "the pages have no data");
        if ((reinterpret_cast<uintptr_t>(g->k) | reinterpret_cast<uintptr_t>(g->v)) & 15u) return fail(TOM_ERR_INVALID_ARG, "the pages must be 16-byte aligned");
        if (!g->rows || (!g->table && g->table_pages > 0)) return fail(TOM_ERR_INVALID_ARG, "table and rows must be non-NULL");
        if ((reinterpret_cast<uintptr_t>(g->table) | reinterpret_cast<uintptr_t>(g->rows) | reinterpret_cast<uintptr_t>(g->starts)) & 3u)
            return fail(TOM_ERR_INVALID_ARG, "table, rows and starts must be 4-byte aligned");
    }
    p.table = g->table;
    p.rows = g->rows;
    p.starts = g->starts;
    p.page_step = (uint32_t)(bytes[1] / 16);
    p.row_step = (uint32_t)(bytes[3] / 16);
    p.head_bytes = bytes[2];
    p.sequences = g->sequences;
    p.table_pages = g->table_pages;
    p.n_pages = g->n_pages;
    p.page_rows = g->page_rows;
    p.inv_page_rows = reciprocal_u32((uint32_t)g->page_rows);
    p.capacity = g->table_pages * g->page_rows;
    return TOM_OK;
}
inline int64_t layer_bytes(const tom_oqm_pages_t& g, int32_t layer) { return layer * g.layer_stride * bytes_of_dtype(g.dtype); }

constexpr uint32_t kNoPlace = 0xffffffffu;  // (a place is below 2^32 - 64)

// Where row `row` of a sequence of `rows` rows (at most the capacity) is; `table`: the sequence's.
__device__ __forceinline__ uint32_t place_of(const PagePlaces& p, const int32_t* table, uint32_t row, uint32_t rows) {
    if (row >= rows) return kNoPlace;
    const uint32_t i = div_by(row, (uint32_t)p.page_rows, p.inv_page_rows);
    const int32_t page = table[i];
    if ((uint32_t)page >= (uint32_t)p.n_pages) return kNoPlace;
    return (uint32_t)page * p.page_step + (row - i * (uint32_t)p.page_rows) * p.row_step;
}
// The first token of sequence s, cut to the call's.
__device__ __forceinline__ int32_t start_of(const PagePlaces& p, int32_t s) {
    return p.starts ? min(max(p.starts[s], 0), p.tokens) : min(s, p.tokens);
}
__device__ __forceinline__ int32_t rows_of(const PagePlaces& p, int32_t s) { return min(max(p.rows[s], 0), p.capacity); }
// Whose token it is: the last sequence that starts at or in front of it, -1 where that has ended before (which with ascending starts is
// nobody's).
__device__ __forceinline__ int32_t sequence_of(const PagePlaces& p, int32_t token) {
    if (!p.starts) return token < p.sequences ? token : -1;
    int32_t lo = 0, hi = p.sequences;  // starts[lo] <= token (or lo is 0) and starts[hi] > token (or hi is the last)
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (p.starts[mid] <= token) lo = mid;
        else hi = mid;
    }
    return lo < p.sequences && token >= start_of(p, lo) && token < start_of(p, lo + 1) ? lo : -1;
}

}  // namespace oqm
