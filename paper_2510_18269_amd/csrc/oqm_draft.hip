// What a draft needs around the attention: the tree's masks and positions before it, the accepted rows' move after it.
#include "oqm_pages.h"

namespace oqm {

struct TreeArgs {
    const int32_t* parents;
    PagePlaces seq;  // starts, sequences and tokens alone
    int64_t* mask;
    const int64_t* first;
    int64_t* positions;
    int32_t words;
};

// A token's ancestors are looked for 64 tokens at a time.  A wave closes its 64 among themselves: with each token's own bit and its parent's number (its own where that
// lies further back), six rounds of "take the ancestor's bits, then its ancestor" reach all.  What is left is a walk over the token's blocks, a word each: the bits of where it stands, then the parent
// of the highest of them, which lies in an earlier block.  96 drafts of 5 to 200 tokens, us: a walk of a token at a time, some 45 dependent reads, 10.5; by blocks 3.3.
// Tokens that have no mask bit for themselves, from 4096 on, walk a token at a time until they come to those that do: a chain of 65536 takes 54 ms with 64 words, by
// 16 workgroups, and 0.81 s with up to 4, by one.
constexpr int kTreeBlock = 256, kStaged = 4096, kMostDrafted = 1 << 16;
__global__ __launch_bounds__(kTreeBlock) void draft_tree_kernel(TreeArgs g) {
    __shared__ uint64_t bits_of[kStaged];
    __shared__ int32_t parent_of[kStaged];  // of the highest of a token's ancestors in its block; -1: none
    const int32_t s = (int32_t)blockIdx.x;
    const int32_t begin = start_of(g.seq, s), count = min(start_of(g.seq, s + 1) - begin, kMostDrafted);
    const int32_t lane = (int32_t)(threadIdx.x & 63), wave = (int32_t)(threadIdx.x >> 6);
    const int32_t* const parents = g.parents + begin;
    auto parent = [&](int32_t t) {
        const int32_t p = parents[t];
        return p < t ? max(p, -1) : -1;
    };
    int32_t closed = 0;
    for (int32_t first = (int32_t)blockIdx.y * kTreeBlock; first < count; first += (int32_t)gridDim.y * kTreeBlock) {
        const int32_t end = min(min(first + kTreeBlock, count), kStaged);
        for (int32_t t0 = closed + 64 * wave; t0 < end; t0 += kTreeBlock) {
            const int32_t t = t0 + lane, p = t < count ? parent(t) : -1;
            int32_t top = p >= t0 ? p - t0 : lane;
            uint64_t bits = uint64_t{1} << lane;
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                bits |= (uint64_t)__shfl((unsigned long long)bits, top, 64);
                top = __shfl(top, top, 64);
            }
            const int32_t out = __shfl(p >= t0 ? -1 : p, top, 64);
            bits_of[t] = bits;  // (kStaged is a multiple of 64)
            parent_of[t] = out;
        }
        closed = max(closed, (end + kTreeBlock - 1) / kTreeBlock * kTreeBlock);
        __syncthreads();
        const int32_t own = first + (int32_t)threadIdx.x;
        if (own < count) {
            const int64_t token = begin + own;
            uint64_t* const mask = reinterpret_cast<uint64_t*>(g.mask) + token * g.words;
            int32_t word = g.words - 1, at = own, seen = 0;
            uint64_t bits = 0;
            auto leave = [&](int32_t to) {  // the words behind `to` are complete
                for (; word > to; --word) {
                    mask[word] = bits;
                    bits = 0;
                }
            };
            for (; at >= kStaged; at = parent(at)) {  // one at a time: there is no room for so many
                leave(at / 64);
                if (at / 64 == word) bits |= uint64_t{1} << (at % 64);
                ++seen;
            }
            while (at >= 0) {
                leave(at / 64);
                const uint64_t more = bits_of[at];
                if (at / 64 == word) bits |= more;
                seen += __popcll(more);
                at = parent_of[at];
            }
            leave(-1);
            if (g.positions) g.positions[token] = (g.first ? g.first[s] : 0) + seen - 1;
        }
        __syncthreads();
    }
}

struct KeepArgs {
    char *k, *v;
    PagePlaces p;
    int64_t layer_bytes;
    const int32_t* idx;
    const int32_t* counts;
    int32_t* rows_out;  // NULL: a launch of its own writes them
    int32_t width, heads;
    uint32_t cols, inv_cols, planes;  // 16 bytes of a row; layers * heads * 2
    uint32_t blocks_per_sequence, inv_blocks;
    uint32_t inv_heads;
};

// A workgroup has 16-byte columns of rows of one sequence, a lane each (of one layer, head and of K or V).  Where the list's rows are is looked up by all its lanes at once; then a
// lane walks the list from the front: kAhead pieces are read, then written.  The list ascends, so idx[i] >= i, and what a batch writes lies in front of all that
// later batches read: in place without a second copy, and no lane touches another's column.  64 sequences of up to 12 kept rows in 28 layers (44 MB), us: every row
// looked up on the way by the wave 15.9, as it is 8.5.
constexpr int kAhead = 8;
// How many rows a sequence then has: all that it had count, those behind the table's end too.
__device__ __forceinline__ int32_t rows_kept(const KeepArgs& g, int32_t s) {
    return (int32_t)min((int64_t)max(g.p.rows[s], 0) + min(max(g.counts[s], 0), g.width), (int64_t)0x7fffffff);
}
__global__ __launch_bounds__(kBlock) void keep_rows_kernel(KeepArgs g) {
    __shared__ uint32_t source_of[kBlock], to_of[kBlock];
    const uint32_t s = div_by(blockIdx.x, g.blocks_per_sequence, g.inv_blocks), block = blockIdx.x - s * g.blocks_per_sequence;
    const uint32_t i = block * kBlock + threadIdx.x, plane = div_by(i, g.cols, g.inv_cols), col = i - plane * g.cols;
    const int32_t rows = rows_of(g.p, (int32_t)s), count = min(max(g.counts[s], 0), g.width);
    if (g.rows_out && i == 0) g.rows_out[s] = rows_kept(g, (int32_t)s);
    const int32_t own = start_of(g.p, (int32_t)s + 1) - start_of(g.p, (int32_t)s);
    const uint32_t layer_head = plane >> 1, layer = div_by(layer_head, (uint32_t)g.heads, g.inv_heads), head = layer_head - layer * (uint32_t)g.heads;
    char* const base = ((plane & 1) ? g.v : g.k) + layer * g.layer_bytes + head * g.p.head_bytes + (int64_t)col * 16;
    const int32_t* const table = g.p.table + (int64_t)s * g.p.table_pages;
    const int32_t* const idx = g.idx + (int64_t)s * g.width;
    for (int32_t begin = 0; begin < count; begin += kBlock) {
        const int32_t end = min(begin + kBlock, count), at = begin + (int32_t)threadIdx.x;
        if (at < end) {
            const int32_t from = idx[at];
            uint32_t source = kNoPlace, to = kNoPlace;
            if (from > at && from < own && from < g.p.capacity - rows) {  // (else it is in its place, or not there)
                source = place_of(g.p, table, (uint32_t)(rows + from), (uint32_t)g.p.capacity);
                if (source != kNoPlace) to = place_of(g.p, table, (uint32_t)(rows + at), (uint32_t)g.p.capacity);
            }
            source_of[threadIdx.x] = source;
            to_of[threadIdx.x] = to;
        }
        __syncthreads();
        if (plane < g.planes) {
            for (int32_t first = 0; first < end - begin; first += kAhead) {
                u32x4 piece[kAhead];
                uint32_t to[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    to[u] = first + u < end - begin ? to_of[first + u] : kNoPlace;
                    if (to[u] != kNoPlace) piece[u] = *reinterpret_cast<const u32x4*>(base + (int64_t)source_of[first + u] * 16);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (to[u] != kNoPlace) *reinterpret_cast<u32x4*>(base + (int64_t)to[u] * 16) = piece[u];
            }
        }
        __syncthreads();
    }
}
__global__ __launch_bounds__(kBlock) void kept_rows_kernel(KeepArgs g, int32_t* rows_out) {
    const uint32_t s = blockIdx.x * kBlock + threadIdx.x;
    if (s < (uint32_t)g.p.sequences) rows_out[s] = rows_kept(g, (int32_t)s);
}

}  // namespace oqm

using namespace oqm;

extern "C" {

tom_status_t tom_oqm_draft_tree(const int32_t* parents, const int32_t* starts, int32_t sequences, int32_t tokens, int64_t* mask, int32_t words,
                                const int64_t* first, int64_t* positions, void* hip_stream) {
    if (sequences < 0 || tokens < 0) return fail(TOM_ERR_INVALID_ARG, "sequences or tokens is negative");
    if (words < 1 || words > 64) return fail(TOM_ERR_INVALID_ARG, "words = %d must be in [1, 64]", words);
    if (!starts && tokens != sequences) return fail(TOM_ERR_INVALID_ARG, "%d tokens of %d sequences: without starts each has one", tokens, sequences);
    if (sequences > kMaxSequences || tokens > (1 << 24)) return fail(TOM_ERR_UNSUPPORTED, "%d sequences of %d tokens: at most 2^20 and 2^24 per call", sequences, tokens);
    if (sequences == 0 || tokens == 0) return TOM_OK;
    if (!parents || !mask) return fail(TOM_ERR_INVALID_ARG, "parents and mask must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(parents) | reinterpret_cast<uintptr_t>(starts)) & 3u) return fail(TOM_ERR_INVALID_ARG, "parents and starts must be 4-byte aligned");
    if ((reinterpret_cast<uintptr_t>(mask) | reinterpret_cast<uintptr_t>(first) | reinterpret_cast<uintptr_t>(positions)) & 7u)
        return fail(TOM_ERR_INVALID_ARG, "mask, first and positions must be 8-byte aligned");
    TreeArgs g{};
    g.parents = parents;
    g.seq.starts = starts;
    g.seq.sequences = sequences;
    g.seq.tokens = tokens;
    g.mask = mask;
    g.first = first;
    g.positions = positions;
    g.words = words;
    // workgroups of a sequence: one for each 256 tokens that a mask has bits for, few where there are many sequences (they take several blocks of tokens
    // where a sequence has more)
    const int32_t most = (words * 64 + kTreeBlock - 1) / kTreeBlock, want = 4096 / sequences + 1;
    (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
    launch(draft_tree_kernel, dim3((uint32_t)sequences, (uint32_t)(most < want ? most : want)), dim3(kTreeBlock), 0, static_cast<hipStream_t>(hip_stream), g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(TOM_ERR_HIP, "draft_tree launch: %s", hipGetErrorString(e));
    return TOM_OK;
}

tom_status_t tom_oqm_keep_rows(const tom_oqm_pages_t* pages, const int32_t* idx, int32_t width, const int32_t* counts, int32_t* rows_out, void* hip_stream) {
    KeepArgs g{};
    if (tom_status_t st = check_pages(pages, g.p)) return st;
    if (width < 0) return fail(TOM_ERR_INVALID_ARG, "width < 0");
    if (pages->sequences == 0) return TOM_OK;
    if ((!idx && width > 0) || !counts || !rows_out) return fail(TOM_ERR_INVALID_ARG, "idx, counts and rows_out must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(idx) | reinterpret_cast<uintptr_t>(counts) | reinterpret_cast<uintptr_t>(rows_out)) & 3u)
        return fail(TOM_ERR_INVALID_ARG, "idx, counts and rows_out must be 4-byte aligned");
    const uint64_t cols = (uint64_t)pages->channels * bytes_of_dtype(pages->dtype) / 16;
    const __int128 pieces = (__int128)pages->n_layers * pages->heads * 2 * cols;
    if (pieces > 0x7fffffff) return fail(TOM_ERR_UNSUPPORTED, "layers and heads of more than 2^31 - 1 pieces of 16 bytes a row");
    const uint64_t blocks = ((uint64_t)pieces + kBlock - 1) / kBlock;
    if (blocks * (uint64_t)pages->sequences * kBlock > kMaxLanes)
        return fail(TOM_ERR_UNSUPPORTED, "%d sequences need more lanes than the 2^32 - 1 of a launch: keep fewer per call", pages->sequences);
    g.k = static_cast<char*>(pages->k);
    g.v = static_cast<char*>(pages->v);
    g.layer_bytes = pages->n_layers > 1 ? layer_bytes(*pages, 1) : 0;
    g.idx = idx;
    g.counts = counts;
    const bool in_place = rows_out == pages->rows;
    g.rows_out = in_place ? nullptr : rows_out;
    g.width = width;
    g.heads = pages->heads;
    g.inv_heads = reciprocal_u32((uint32_t)pages->heads);
    g.cols = (uint32_t)cols;
    g.inv_cols = reciprocal_u32(g.cols);
    g.planes = (uint32_t)((uint64_t)pieces / cols);
    g.blocks_per_sequence = (uint32_t)blocks;
    g.inv_blocks = reciprocal_u32(g.blocks_per_sequence);
    // how many tokens each sequence has says how far its list may reach; without an end of the call to cut it to
    g.p.tokens = 0x7fffffff;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
    launch(keep_rows_kernel, dim3((uint32_t)(blocks * (uint64_t)pages->sequences)), dim3(kBlock), 0, s, g);
    if (in_place) launch(kept_rows_kernel, dim3((uint32_t)((pages->sequences + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, g, rows_out);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(TOM_ERR_HIP, "keep_rows launch: %s", hipGetErrorString(e));
    return TOM_OK;
}

}  // extern "C"
