// What the kernels of the attention over pages share: which part of which block of query rows a workgroup has, what a token sees, and how
// a row's result is written.
#pragma once

#include "oqm_attend_device.h"
#include "oqm_attend_pages.h"

namespace oqm {

// Lies where a row of a sequence does not: what is not there is read as zero.
static __device__ const u32x4 kZeroRow[64] = {};

struct Block {  // a block of query rows of a sequence, and a part of its rows
    int32_t sequence, first_token, tokens, rows;  // rows: without the call's
    int32_t tile;                                 // which block of the sequence
    int32_t begin, end;                           // rows of the part
    int32_t for_all;                              // rows from the first that all of the block's tokens see
    uint32_t first_item, parts;
};

// Of x items, in LDS: the sequence whose item it is and that one's first, and the length of a part.
struct FoundItem {
    uint32_t x_in_sequence, base, parts;
    int32_t sequence, chunk;
    uint64_t totals[16];
    uint32_t counts[16];
};

template <int QT>
__device__ __forceinline__ uint32_t tiles_of(const PagesArgs& g, int32_t tokens) {
    return ((uint32_t)tokens * (uint32_t)g.repeat + QT - 1) / QT;  // H_q * tokens is below 2^30
}

// How far the last token of a block sees: less for the earlier blocks of a sequence where a token does not see those behind it.
template <int QT>
__device__ __forceinline__ int32_t end_of(const PagesArgs& g, int32_t rows, int32_t tokens, int32_t tile) {
    if (!g.causal || g.mask) return (int32_t)min((int64_t)rows + tokens, (int64_t)g.p.capacity);
    const uint32_t last_row = min((uint32_t)(tile + 1) * QT, (uint32_t)tokens * (uint32_t)g.repeat) - 1;
    return (int32_t)min((int64_t)rows + div_by(last_row, (uint32_t)g.repeat, g.inv_repeat) + 1, (int64_t)g.p.capacity);
}
// Of a sequence's blocks the first that sees `seen` rows or more (their number: none does).
template <int QT>
__device__ __forceinline__ uint32_t first_seeing(const PagesArgs& g, int32_t rows, int32_t tokens, int64_t seen) {
    const uint32_t tiles = tiles_of<QT>(g, tokens);
    if (seen <= 0 || tiles == 0) return 0;
    if (min((int64_t)rows + tokens, (int64_t)g.p.capacity) < seen) return tiles;
    if (!g.causal || g.mask || seen <= rows) return 0;
    // token t (from 1) sees rows + t; block j's last is min(tokens, ((j + 1) QT - 1) / repeat + 1)
    return (uint32_t)(((uint64_t)(seen - rows - 1) * (uint32_t)g.repeat) / QT);
}

// The same in every lane of the workgroup; false: there is nothing for it.
// All workgroups look at all sequences: a sum over them says how long a part is (so that a long sequence among short ones is cut and they are not), a second
// one where each one's items begin; the host knows none of the lengths.  A call without parts (pages_cuts) cuts no sequence, however long one is among the others.
template <int QT, int KT, int THREADS>
__device__ __forceinline__ bool block_of(const PagesArgs& g, uint32_t x, FoundItem& found, Block& b) {
    const int32_t sequences = g.p.sequences;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t in_sequence, base;
    int32_t s, chunk = 0x7fffffff;
    auto part_length = [&](uint64_t total) {  // whole tiles, above total / extra
        return (int32_t)min(max((total / g.extra + KT) / KT * KT, (uint64_t)g.least), (uint64_t)0x7fffffff);
    };
    int32_t first_token = -1, tokens = 0, rows = 0;  // of s, once they are known
    if (sequences == 1) {
        s = 0;
        base = 0;
        const int32_t n = max(start_of(g.p, 1) - start_of(g.p, 0), 0);
        const uint32_t tiles = tiles_of<QT>(g, n);
        in_sequence = x;
        if (g.extra) {
            chunk = part_length((uint64_t)tiles * (uint64_t)min((int64_t)rows_of(g.p, 0) + n, (int64_t)g.p.capacity));
        } else {
            if (x >= tiles) return false;
            in_sequence = tiles - 1 - x;  // the longest first
        }
    } else if (sequences <= 64 && (g.p.starts || g.extra)) {
        // One a lane, in every wave for itself: the same as below without LDS or a barrier, and what a lane has loaded is not loaded again.  4 drafts of 43 to 52 tokens, us,
        // as below 37.6, so 35.9; three prompts 369 / 360; but one sequence 13.2 / 13.7 (and above 13.2).
        const int32_t i = min(lane, sequences - 1), first = start_of(g.p, i), behind = start_of(g.p, i + 1);
        const int32_t had = rows_of(g.p, i), n = lane < sequences ? max(behind - first, 0) : 0;
        const uint32_t tiles = tiles_of<QT>(g, n), all = (uint32_t)min((int64_t)had + n, (int64_t)g.p.capacity);
        uint32_t mine = tiles, level = 0;
        if (g.extra) {
            uint64_t total = (uint64_t)tiles * all;
            for (int m = 32; m > 0; m /= 2) total += __shfl_xor(total, m, 64);
            chunk = part_length(total);
            mine *= max((all + (uint32_t)chunk - 1u) / (uint32_t)chunk, 1u);
        } else if (g.sorted) {
            auto seeing = [&](uint32_t steps) { return tiles - first_seeing<QT>(g, had, n, (int64_t)steps * 64); };
            uint32_t x_from = 0;
            for (uint32_t bit = 1u << (31 - __builtin_clz((uint32_t)g.p.capacity / 64 + 1)); bit > 0; bit /= 2) {
                uint32_t all_seeing = seeing(level + bit);
                for (int m = 32; m > 0; m /= 2) all_seeing += __shfl_xor(all_seeing, m, 64);
                if (all_seeing > x) level += bit;
                else x_from = all_seeing;
            }
            x -= x_from;
            mine = seeing(level) - seeing(level + 1);
        }
        uint32_t before = mine;
        for (int m = 1; m < 64; m *= 2) {
            const uint32_t other = __shfl_up(before, m, 64);
            if (lane >= m) before += other;
        }
        before -= mine;
        const uint64_t hit = __ballot(x >= before && x < before + mine);
        if (!hit) return false;
        s = __builtin_ctzll(hit);
        base = (uint32_t)__builtin_amdgcn_readlane((int)before, s);
        first_token = __builtin_amdgcn_readlane(first, s);
        tokens = __builtin_amdgcn_readlane(n, s);
        rows = __builtin_amdgcn_readlane(had, s);
        in_sequence = x - base;
        if (g.sorted) in_sequence += first_seeing<QT>(g, rows, tokens, (int64_t)level * 64);
    } else if (!g.p.starts && g.extra == 0) {
        const uint32_t tiles = tiles_of<QT>(g, 1);
        s = (int32_t)(x / tiles);
        in_sequence = x - (uint32_t)s * tiles;
        base = (uint32_t)s * tiles;
    } else if (!g.extra && sequences > kMostSorted) {
        // (a look at all of them by every workgroup would cost more than their order gives: x counts units, which some are nobody's of)
        auto first_unit = [&](int32_t i) {
            const int32_t at = start_of(g.p, i);
            return (uint32_t)at * (uint32_t)g.repeat / QT + (uint32_t)min(i, at);
        };
        int32_t hi = sequences;  // the last that begins at or in front of x
        s = 0;
        while (hi - s > 1) {
            const int32_t mid = (s + hi) >> 1;
            if (first_unit(mid) <= x) s = mid;
            else hi = mid;
        }
        base = first_unit(s);
        in_sequence = x - base;
    } else {
        const int32_t per = (sequences + THREADS - 1) / THREADS, from = min(tid * per, sequences), to = min(from + per, sequences);
        auto shape = [&](int32_t i, uint32_t& tiles, uint32_t& rows) {
            const int32_t n = max(start_of(g.p, i + 1) - start_of(g.p, i), 0);
            tiles = tiles_of<QT>(g, n);
            rows = (uint32_t)min((int64_t)rows_of(g.p, i) + n, (int64_t)g.p.capacity);
        };
        if (g.extra) {
            uint64_t total = 0;
            for (int32_t i = from; i < to; ++i) {
                uint32_t tiles, rows;
                shape(i, tiles, rows);
                total += (uint64_t)tiles * rows;
            }
            for (int m = 32; m > 0; m /= 2) total += __shfl_xor(total, m, 64);
            if (lane == 0) found.totals[wave] = total;
            __syncthreads();
            total = 0;
            for (int w = 0; w < THREADS / 64; ++w) total += found.totals[w];
            chunk = part_length(total);
        }
        // More blocks than run at a time go by what they see, in steps of 64 rows, the longest first, so that none is left to run alone at the end: that many of them
        // see `level` steps and more, and x counts on from those that see a step more.
        int32_t level = 0;
        uint32_t x_from = 0;
        auto seeing = [&](int32_t i, int32_t steps) {
            const int32_t n = max(start_of(g.p, i + 1) - start_of(g.p, i), 0);
            return tiles_of<QT>(g, n) - first_seeing<QT>(g, rows_of(g.p, i), n, (int64_t)steps * 64);
        };
        if (g.sorted) {
            for (int32_t bit = 1 << (31 - __builtin_clz((uint32_t)g.p.capacity / 64 + 1)); bit > 0; bit /= 2) {
                uint32_t mine = 0;
                for (int32_t i = from; i < to; ++i) mine += seeing(i, level + bit);
                for (int m = 32; m > 0; m /= 2) mine += __shfl_xor(mine, m, 64);
                if (lane == 0) found.counts[wave] = mine;
                __syncthreads();
                uint32_t all = 0;
                for (int w = 0; w < THREADS / 64; ++w) all += found.counts[w];
                __syncthreads();
                if (all > x) level += bit;
                else x_from = all;  // (the counts fall as levels rise: the last of these is that of one level more)
            }
            x -= x_from;
        }
        auto items = [&](int32_t i) {
            if (g.sorted) return seeing(i, level) - seeing(i, level + 1);
            uint32_t tiles, rows;
            shape(i, tiles, rows);
            return tiles * max((rows + (uint32_t)chunk - 1u) / (uint32_t)chunk, 1u);
        };
        uint32_t mine = 0;
        for (int32_t i = from; i < to; ++i) mine += items(i);
        uint32_t before = mine;
        for (int m = 1; m < 64; m *= 2) {
            const uint32_t other = __shfl_up(before, m, 64);
            if (lane >= m) before += other;
        }
        if (lane == 63) found.counts[wave] = before;
        if (tid == 0) found.sequence = -1;
        before -= mine;
        __syncthreads();
        for (int w = 0; w < wave; ++w) before += found.counts[w];
        if (x >= before && x < before + mine) {
            int32_t i = from;
            uint32_t at = before, n = items(i);
            while (x >= at + n) {
                at += n;
                n = items(++i);
            }
            found.sequence = i;
            found.base = at;
        }
        __syncthreads();
        s = found.sequence;
        if (s < 0) return false;
        base = found.base;
        in_sequence = x - base;
        if (g.sorted) {
            const int32_t n = max(start_of(g.p, s + 1) - start_of(g.p, s), 0);
            in_sequence += first_seeing<QT>(g, rows_of(g.p, s), n, (int64_t)level * 64);
        }
    }
    s = __builtin_amdgcn_readfirstlane(s);
    if (first_token < 0) {
        first_token = start_of(g.p, s);
        tokens = max(start_of(g.p, s + 1) - first_token, 0);
        rows = rows_of(g.p, s);
    }
    b.sequence = s;
    b.first_token = first_token;
    b.tokens = tokens;
    b.rows = rows;
    const int32_t all = (int32_t)min((int64_t)b.rows + b.tokens, (int64_t)g.p.capacity);
    b.parts = g.extra ? max(((uint32_t)all + (uint32_t)chunk - 1u) / (uint32_t)chunk, 1u) : 1u;
    b.tile = (int32_t)(in_sequence / b.parts);
    const uint32_t part = in_sequence - (uint32_t)b.tile * b.parts;
    if ((uint32_t)b.tile >= tiles_of<QT>(g, b.tokens)) return false;
    b.first_item = base + (uint32_t)b.tile * b.parts;
    b.begin = 0;
    b.end = all;
    if (b.parts > 1) {
        b.begin = (int32_t)part * chunk;
        b.end = (int32_t)min((uint32_t)all, (uint32_t)b.begin + (uint32_t)chunk);
    }
    b.end = min(b.end, end_of<QT>(g, b.rows, b.tokens, b.tile));
    b.for_all = b.rows;
    if (!g.mask) b.for_all = !g.causal ? all : (int32_t)min((int64_t)b.rows + div_by((uint32_t)b.tile * QT, (uint32_t)g.repeat, g.inv_repeat) + 1, (int64_t)all);
    // the same in all lanes, which the compiler cannot see of what has gone through LDS
    for (int32_t* x : {&b.first_token, &b.tokens, &b.rows, &b.tile, &b.begin, &b.end, &b.for_all}) *x = __builtin_amdgcn_readfirstlane(*x);
    b.first_item = (uint32_t)__builtin_amdgcn_readfirstlane((int)b.first_item);
    b.parts = (uint32_t)__builtin_amdgcn_readfirstlane((int)b.parts);
    return true;
}
// Where a block's first item and its parts stand: unique, and below the units that the host counts.  (A sequence with tokens has as many in front of
// it as it has predecessors with some, at most.)
template <int QT>
__device__ __forceinline__ uint32_t unit_of(const PagesArgs& g, int32_t s, int32_t first_token, int32_t tile) {
    if (!g.p.starts) return (uint32_t)s * tiles_of<QT>(g, 1) + (uint32_t)tile;
    return (uint32_t)first_token * (uint32_t)g.repeat / QT + (uint32_t)min(s, first_token) + (uint32_t)tile;
}

// For the join: where a block's items begin, and how many they are.
template <int QT>
__device__ __forceinline__ void tell_unit(const PagesArgs& g, const Block& b, uint32_t x, int head) {
    if (g.extra == 0 || head != 0 || x != b.first_item || threadIdx.x != 0) return;
    uint32_t* const unit = g.unit_first + 2 * (size_t)unit_of<QT>(g, b.sequence, b.first_token, b.tile);
    unit[0] = b.first_item;
    unit[1] = b.parts;
}

// Of the N rows (32 or 64) from t0 those that token `own` of a sequence sees, as bits; what lies behind the sequence's rows is left to the caller.
template <int N>
__device__ __forceinline__ uint64_t seen_from(const PagesArgs& g, int32_t t0, int32_t rows, int32_t own, const uint64_t* mask) {
    const int32_t at = t0 - rows;  // of the call's tokens; |t0|, |rows| < 2^31
    if (at <= -N) return ~uint64_t{0};
    if (mask) {
        if (at < 0) return mask[0] << -at | ((uint64_t{1} << -at) - 1);
        const int32_t w = at >> 6, up = at & 63;
        uint64_t bits = w < g.words ? mask[w] >> up : 0;
        if (up && w + 1 < g.words) bits |= mask[w + 1] << (64 - up);
        return bits;
    }
    if (!g.causal) return ~uint64_t{0};
    const int32_t count = own + 1 - at;  // (at > -64, own < 2^20)
    return count >= 64 ? ~uint64_t{0} : count <= 0 ? 0 : (uint64_t{1} << count) - 1;
}

// Values that are not finite (an exponent of all ones), by their bits: the build assumes that arithmetic meets no NaN.  Of a word, in one of its halves
// or (float32) in all of it.
template <typename T>
__device__ __forceinline__ bool any_odd(uint32_t w) {
    constexpr uint32_t m = __is_same(T, In_f32) ? 0x7f800000u : __is_same(T, In_bf16) ? 0x7f80u : 0x7c00u;
    if constexpr (__is_same(T, In_f32)) return (w & m) == m;
    else return (w & m) == m || (w & m << 16) == m << 16;
}
// The word with zeros in their places.
template <typename T>
__device__ __forceinline__ uint32_t without_odd(uint32_t w) {
    constexpr uint32_t m = __is_same(T, In_f32) ? 0x7f800000u : __is_same(T, In_bf16) ? 0x7f80u : 0x7c00u;
    if constexpr (__is_same(T, In_f32)) return (w & m) == m ? 0u : w;
    else return w & (((w & m) == m ? 0u : 0xffffu) | ((w & m << 16) == m << 16 ? 0u : 0xffff0000u));
}

// How a row's sums, counted from `from` (units of log 2), become its result, the prior taken in: out = sums * mine + prior * theirs.
struct RowEnd {
    float mine, theirs, lse;
};
__device__ __forceinline__ RowEnd row_end(const PagesArgs& g, int32_t q_head, int32_t token, float from, float total) {
    float mine = 1.0f, theirs = 0.0f;
    if (g.prior_lse) {
        const float before = g.prior_lse[q_head * g.prior_lse_head + token * g.prior_lse_row] * kLog2e;
        if (before > -__builtin_inff()) {
            const float top = fmaxf(from, before);
            mine = exp2_of(from - top);
            theirs = exp2_of(before - top);
            from = top;
            total = total > 0.0f ? total * mine + theirs : theirs;
        }
    }
    const float by = total > 0.0f ? 1.0f / total : 0.0f;
    return {mine * by, theirs * by, total > 0.0f ? (from + __builtin_amdgcn_logf(total)) * kLn2 : -__builtin_inff()};
}
template <typename T>
__device__ __forceinline__ void put_channels(const PagesArgs& g, int32_t q_head, int32_t token, int c, f32x4 sum, const RowEnd& end) {
    typedef typename Element<T>::type E;
    typedef E Vec __attribute__((ext_vector_type(4)));
    sum *= end.mine;
    // Whether there is a prior is asked of the call, not of the weight: without one that is 0 * (1 / total), and no number where the total is none.
    if (g.prior_out && end.theirs != 0.0f) {
        const Vec x = *reinterpret_cast<const Vec*>(g.prior_out + q_head * g.prior_head + token * g.prior_row + (int64_t)c * sizeof(E));
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(end.theirs, (float)x[i], sum[i]);
    }
    Vec y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (E)sum[i];
    *reinterpret_cast<Vec*>(g.out + q_head * g.out_head + token * g.out_row + (int64_t)c * sizeof(E)) = y;
}
// A row's lanes are of one wave and have all read the prior's sum before the row's own is written, so that both may be one array.
__device__ __forceinline__ void put_lse(const PagesArgs& g, int32_t q_head, int32_t token, const RowEnd& end) {
    if (g.lse) g.lse[q_head * g.lse_head + token * g.lse_row] = end.lse;
}

// Lanes below which a workgroup a row joins them.  (One lane a row takes its 99 parts one after the other: 33 us of a token's call, with a workgroup 6.)
constexpr uint64_t kWideJoin = 48 * 1024;
// Parts joined, four channels of a row a lane: all of them by one lane, or (WIDE) a workgroup a row, whose sets of lanes take the parts in turn and then join what
// they have found, the loads of 16 parts on their way together.  A token of 28 heads over 12.6 K rows (99 parts), us of both launches, by 4 / 8 / 16 parts: 14.3 / 13.9 / 13.3;
// over 500 rows (4 parts) 9.5 / 9.8 / 9.9.
struct JoinedRow {
    float from = -__builtin_inff(), total = 0.0f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float their_from, float their_total, f32x4 their_sum) {
        const float top = fmaxf(from, their_from), base = top == -__builtin_inff() ? 0.0f : top;
        const float mine = exp2_of(from - base), theirs = exp2_of(their_from - base);
        from = top;
        total = total * mine + their_total * theirs;
        sum = sum * mine + their_sum * theirs;
    }
};
template <typename T, int QT, bool WIDE>
__global__ __launch_bounds__(kBlock) void join_pages_kernel(PagesArgs g, uint32_t lanes_log2, uint32_t rows, uint32_t inv_heads_all) {
    const uint32_t lanes = 1u << lanes_log2, lane = threadIdx.x & (lanes - 1);
    const uint32_t sets = WIDE ? kBlock >> lanes_log2 : 1u, set = WIDE ? threadIdx.x >> lanes_log2 : 0u;
    const uint32_t row = WIDE ? blockIdx.x : (blockIdx.x * kBlock + threadIdx.x) >> lanes_log2;
    if (row >= rows) return;
    const uint32_t heads = (uint32_t)(g.kv_heads * g.repeat), token = div_by(row, heads, inv_heads_all), q_head = row - token * heads;
    const int32_t s = sequence_of(g.p, (int32_t)token);
    if (s < 0) return;
    const int32_t first_token = start_of(g.p, s);
    const uint32_t head = div_by(q_head, (uint32_t)g.repeat, g.inv_repeat);
    const uint32_t at = (token - (uint32_t)first_token) * (uint32_t)g.repeat + (q_head - head * (uint32_t)g.repeat);
    const uint32_t* const unit = g.unit_first + 2 * (size_t)unit_of<QT>(g, s, first_token, (int32_t)(at / QT));
    const uint32_t first = unit[0], parts = min(unit[1], first < g.items ? g.items - first : 0u);  // (starts that overlap leave units that nobody has written)
    if (parts <= 1) return;
    const int c = 4 * (int)lane, from_c = c < g.channels ? c : 0;
    const size_t step = (size_t)g.kv_heads * QT;
    const size_t slot = ((size_t)first * g.kv_heads + head) * QT + at % QT;
    const f32pair* const stat = g.part_stat + slot;
    const float* const part = g.part_out + slot * g.channels + from_c;
    constexpr int kAhead = WIDE ? 16 : 4;
    const uint32_t some = WIDE ? (uint32_t)__builtin_amdgcn_readfirstlane((int)parts) : parts;
    JoinedRow j;
    for (uint32_t p0 = set; p0 < parts; p0 += sets * kAhead) {
        f32pair st[kAhead];
        f32x4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (WIDE && u > 0 && u % 4 == 0 && p0 - set + u * sets >= some) break;
            const size_t n = min(p0 + u * sets, parts - 1) * step;  // behind the last: read again, and not added
            st[u] = stat[n];
            x[u] = *reinterpret_cast<const f32x4*>(part + n * g.channels);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (p0 + u * sets < parts) j.add(st[u].x, st[u].y, x[u]);
    }
    if constexpr (WIDE) {
        __shared__ f32pair stats[kBlock];
        __shared__ f32x4 sums[kBlock];
        stats[threadIdx.x] = f32pair{j.from, j.total};
        sums[threadIdx.x] = j.sum;
        __syncthreads();
        if (set > 0) return;
        for (uint32_t i = 1; i < sets; ++i) j.add(stats[i * lanes + lane].x, stats[i * lanes + lane].y, sums[i * lanes + lane]);
    }
    if (c >= g.channels) return;
    const RowEnd end = row_end(g, (int32_t)q_head, (int32_t)token, j.from, j.total);
    put_channels<T>(g, (int32_t)q_head, (int32_t)token, c, j.sum, end);
    if (c == 0) put_lse(g, (int32_t)q_head, (int32_t)token, end);
}
template <typename T, int QT>
void start_join_pages(const PagesArgs& g, hipStream_t s) {
    const uint32_t heads = (uint32_t)(g.kv_heads * g.repeat), rows = heads * (uint32_t)g.p.tokens;  // (calls with parts have less than 2^20 rows)
    const uint32_t lanes_log2 = g.channels <= 64 ? 4 : g.channels <= 128 ? 5 : 6;
    if ((uint64_t)rows << lanes_log2 < kWideJoin) launch(join_pages_kernel<T, QT, true>, dim3(rows), dim3(kBlock), 0, s, g, lanes_log2, rows, reciprocal_u32(heads));
    else launch(join_pages_kernel<T, QT, false>, dim3((uint32_t)((((uint64_t)rows << lanes_log2) + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, g, lanes_log2, rows, reciprocal_u32(heads));
}

}  // namespace oqm
