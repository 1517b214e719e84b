// Groups of a memory moved as they are stored: a chosen few kept, the others dropped (in place), or copied to the end of
// another memory.  Nothing is computed: a pass reads and writes every byte of the groups once, and memory bounds it.
#include "oqm_common.h"

namespace oqm {

// One of the storage arrays: `planes` planes of slots of `cols` pieces of the launch's piece size.
struct GroupArray {
    const char* from;
    char* to;
    int64_t from_plane, to_plane, slot_bytes;  // bytes between two planes, of a slot
    uint32_t cols;
    uint32_t col_log2;             // columns a workgroup takes: 2^col_log2
    uint32_t col_blocks;           // workgroups over the columns of a plane
    uint32_t first_block;          // of this array in the grid
};
struct GroupArgs {
    GroupArray a[3];  // codes, meta, keys
    const int32_t* idx;
    int32_t n, n_groups, first_slot;
    uint32_t rows_per_block;  // of the list; a multiple of what a workgroup has in flight unless it is all of it
};

// A workgroup holds a strip of columns of a plane and walks its part of the list from the front: kAhead pieces a lane are read,
// then written.  In place (the list ascends, so idx[i] >= i) this needs no second copy of anything: a strip belongs to one
// workgroup, which writes slot i only after every list entry up to the end of its batch has been read, and later batches read
// slots from their own position in the list up, which no earlier batch writes.  Where a lane has its column to itself nobody else
// touches it, and the wave's own order is enough.
// 96 of 128 groups of 196 tokens in 28 layers kept (685 MB), us: workgroups of 256 lanes with a barrier in every batch 142 (8
// pieces), 168 (4), 198 (16); without 131; of 128 lanes 128.5; of 64 125.8 = 5.4 TB/s; the same with loads past the caches 134,
// with stores that stay in them 141.
constexpr int kAhead = 8;
template <typename PIECE, bool IN_PLACE>
__global__ __launch_bounds__(1024) void move_groups_kernel(GroupArgs g) {
    uint32_t w = 0;
    if (blockIdx.x >= g.a[1].first_block) w = 1;
    if (blockIdx.x >= g.a[2].first_block) w = 2;
    const GroupArray a = w == 0 ? g.a[0] : w == 1 ? g.a[1] : g.a[2];
    const uint32_t block = blockIdx.x - a.first_block;
    const uint32_t plane = block / a.col_blocks, strip = block % a.col_blocks;
    const uint32_t col = (strip << a.col_log2) + (threadIdx.x & ((1u << a.col_log2) - 1u));
    const uint32_t rows = blockDim.x >> a.col_log2;  // of the list at a time
    const bool there = col < a.cols;
    const char* from = a.from + plane * a.from_plane + (int64_t)col * sizeof(PIECE);
    char* to = a.to + plane * a.to_plane + (int64_t)col * sizeof(PIECE);
    const int64_t begin = (int64_t)blockIdx.y * g.rows_per_block;
    const int64_t end = min((int64_t)g.n, begin + g.rows_per_block);
    for (int64_t r0 = begin; r0 < end; r0 += rows * kAhead) {
        const int64_t first = r0 + (threadIdx.x >> a.col_log2);
        PIECE piece[kAhead];
        bool moves[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t r = first + u * rows;
            int32_t slot = -1;
            if (there && r < end) slot = g.idx[r];
            moves[u] = slot >= 0 && slot < g.n_groups && !(IN_PLACE && slot == r);
            if (moves[u]) piece[u] = *reinterpret_cast<const PIECE*>(from + (int64_t)slot * a.slot_bytes);
        }
        if (IN_PLACE && rows > 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what other lanes are about to overwrite has arrived
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t r = first + u * rows;
            if (moves[u]) __builtin_nontemporal_store(piece[u], reinterpret_cast<PIECE*>(to + (int64_t)(g.first_slot + r) * a.slot_bytes));
        }
    }
}

typedef uint32_t piece16 __attribute__((ext_vector_type(4)));
typedef uint64_t piece8;

template <bool IN_PLACE>
hipError_t launch_move_groups(const tom_oqm_t& to, const tom_oqm_t& from, const int32_t* idx, int32_t n, int32_t first_slot, hipStream_t s) {
    const tom_oqm_config_t& c = from.cfg;
    const Layout lay = layout_of(c);
    GroupArgs g{};
    g.idx = idx;
    g.n = n;
    g.n_groups = from.n_groups;
    g.first_slot = first_slot;
    const uint64_t bytes[3] = {(uint64_t)c.n_kv_heads * lay.tile_code_bytes,
                               (uint64_t)c.n_kv_heads * lay.tile_meta * (c.meta_dtype == TOM_BF16 ? 4 : 8),
                               (uint64_t)c.n_kv_heads * c.head_dim * sizeof(float)};
    const char* const src[3] = {reinterpret_cast<const char*>(from.codes), static_cast<const char*>(from.meta), reinterpret_cast<const char*>(from.keys)};
    char* const dst[3] = {reinterpret_cast<char*>(to.codes), static_cast<char*>(to.meta), reinterpret_cast<char*>(to.keys)};
    // The widest piece that divides a slot of every array (arrays start on 16 bytes): codes of 2 bits and 8 channels leave 2 bytes.
    const uint64_t all = bytes[0] | bytes[1] | bytes[2];
    const uint32_t piece = all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : 2;
    // In place, strips that are too few to fill the chip are walked by more lanes at a time: 1024 in a workgroup, on strips as narrow as
    // the list needs to be read in one batch, but no narrower than 16 pieces.
    uint32_t threads = 64, widest = 6;
    if (IN_PLACE) {
        uint64_t waves = 0;
        for (int i = 0; i < 3; ++i) waves += (uint64_t)c.n_layers * (i < 2 ? 2 : 1) * ((bytes[i] / piece + 63) / 64);
        if (waves < 1024 && n > kAhead) {
            threads = 1024;
            while (widest > 4 && (int64_t)(1024u >> widest) * kAhead < n) --widest;
        }
    }
    uint64_t blocks = 0;
    for (int i = 0; i < 3; ++i) {
        GroupArray& a = g.a[i];
        const uint64_t planes = (uint64_t)c.n_layers * (i < 2 ? 2 : 1);
        a.from = src[i];
        a.to = dst[i];
        a.slot_bytes = (int64_t)bytes[i];
        a.from_plane = (int64_t)bytes[i] * from.cfg.capacity_groups;
        a.to_plane = (int64_t)bytes[i] * to.cfg.capacity_groups;
        if (bytes[i] / piece > 0x7fffffffu) return hipErrorInvalidConfiguration;
        a.cols = (uint32_t)(bytes[i] / piece);
        while (a.col_log2 < widest && (1u << a.col_log2) < a.cols) ++a.col_log2;
        a.col_blocks = (a.cols + (1u << a.col_log2) - 1) >> a.col_log2;
        a.first_block = (uint32_t)blocks;
        blocks += planes * a.col_blocks;
        if (blocks > 0x7fffffffu) return hipErrorInvalidConfiguration;
    }
    uint32_t parts = 1;
    g.rows_per_block = (uint32_t)n;
    if (!IN_PLACE) {  // the list may be cut: one batch of the widest strips a workgroup
        g.rows_per_block = kAhead;
        while (((uint32_t)n + g.rows_per_block - 1) / g.rows_per_block > 65535u) g.rows_per_block *= 2;
        parts = ((uint32_t)n + g.rows_per_block - 1) / g.rows_per_block;
    }
    const dim3 grid((uint32_t)blocks, parts), block(threads);
    if (piece == 16) launch(move_groups_kernel<piece16, IN_PLACE>, grid, block, 0, s, g);
    else if (piece == 8) launch(move_groups_kernel<piece8, IN_PLACE>, grid, block, 0, s, g);
    else if (piece == 4) launch(move_groups_kernel<uint32_t, IN_PLACE>, grid, block, 0, s, g);
    else launch(move_groups_kernel<uint16_t, IN_PLACE>, grid, block, 0, s, g);
    return hipGetLastError();
}

// Two memories whose arrays share memory without being the same arrays of the same capacity.
static bool clash(const tom_oqm_t& x, const tom_oqm_t& y) {
    tom_oqm_sizes_t sx, sy;
    if (tom_oqm_query_sizes(&x.cfg, &sx) != TOM_OK || tom_oqm_query_sizes(&y.cfg, &sy) != TOM_OK) return true;
    if (x.codes == y.codes && x.meta == y.meta && x.keys == y.keys && x.cfg.capacity_groups == y.cfg.capacity_groups) return false;
    const uintptr_t px[3] = {reinterpret_cast<uintptr_t>(x.codes), reinterpret_cast<uintptr_t>(x.meta), reinterpret_cast<uintptr_t>(x.keys)};
    const uintptr_t py[3] = {reinterpret_cast<uintptr_t>(y.codes), reinterpret_cast<uintptr_t>(y.meta), reinterpret_cast<uintptr_t>(y.keys)};
    const size_t bx[3] = {sx.codes, sx.meta, sx.keys}, by[3] = {sy.codes, sy.meta, sy.keys};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j)
            if (px[i] < py[j] + by[j] && py[j] < px[i] + bx[i]) return true;
    return false;
}

}  // namespace oqm

using namespace oqm;

extern "C" {

tom_status_t tom_oqm_keep_groups(tom_oqm_t* h, const int32_t* idx, int32_t n, void* hip_stream) {
    if (!h) return fail(TOM_ERR_INVALID_ARG, "handle is NULL");
    if (!h->bound) return fail(TOM_ERR_NOT_BOUND, "tom_oqm_bind has not been called");
    if (n < 0 || n > h->n_groups) return fail(TOM_ERR_INVALID_ARG, "n = %d is outside [0, stored groups = %d]", n, h->n_groups);
    if (n > 0) {
        if (!idx) return fail(TOM_ERR_INVALID_ARG, "idx must be non-NULL");
        if ((reinterpret_cast<uintptr_t>(idx) & 3u) != 0) return fail(TOM_ERR_INVALID_ARG, "idx must be 4-byte aligned");
        (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
        const hipError_t e = launch_move_groups<true>(*h, *h, idx, n, 0, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail(TOM_ERR_HIP, "keep_groups launch: %s", hipGetErrorString(e));
    }
    h->n_groups = n;
    return TOM_OK;
}

tom_status_t tom_oqm_copy_groups(tom_oqm_t* to, const tom_oqm_t* from, const int32_t* idx, int32_t n, void* hip_stream) {
    if (!to || !from) return fail(TOM_ERR_INVALID_ARG, "handle is NULL");
    if (!to->bound || !from->bound) return fail(TOM_ERR_NOT_BOUND, "tom_oqm_bind has not been called");
    if (n < 0) return fail(TOM_ERR_INVALID_ARG, "n < 0");
    const tom_oqm_config_t &a = to->cfg, &b = from->cfg;
    if (a.n_layers != b.n_layers || a.n_kv_heads != b.n_kv_heads || a.head_dim != b.head_dim || a.group_tokens != b.group_tokens ||
        a.bits != b.bits || a.qaxis != b.qaxis || a.meta_dtype != b.meta_dtype || (a.qaxis == TOM_QAXIS_HEAD_DIM && a.qgroup != b.qgroup))
        return fail(TOM_ERR_INVALID_ARG, "the two memories store groups of different shapes");
    if ((int64_t)to->n_groups + n > a.capacity_groups)
        return fail(TOM_ERR_CAPACITY, "%d stored + %d copied frame-groups exceed capacity %d", to->n_groups, n, a.capacity_groups);
    if (n == 0) return TOM_OK;
    if (!idx) return fail(TOM_ERR_INVALID_ARG, "idx must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(idx) & 3u) != 0) return fail(TOM_ERR_INVALID_ARG, "idx must be 4-byte aligned");
    // Two handles on one storage: what the other holds past this one's groups would be read while it is written.
    if (to != from && (clash(*to, *from) || (to->codes == from->codes && from->n_groups > to->n_groups)))
        return fail(TOM_ERR_INVALID_ARG, "the two memories' storage overlaps");
    (void)hipGetLastError();
    const hipError_t e = launch_move_groups<false>(*to, *from, idx, n, to->n_groups, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(TOM_ERR_HIP, "copy_groups launch: %s", hipGetErrorString(e));
    to->n_groups += n;
    return TOM_OK;
}

}  // extern "C"
