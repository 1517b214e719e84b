// Attention of many query rows over codes of any layout: a tile of 32 tokens is reconstructed once in LDS, in 16-bit parts, for
// all the query rows of a workgroup.
//
// In LDS the operands lie as the matrix cores take them, 16 bytes a lane:
//   keys    [half][step][lane][8 channels]       lane = (token of the half, quarter of the channels)
//   values  [block of channels][lane][8 tokens]  lane = (channel of the block, quarter of the tokens)
// Eight waves of 32 rows (of 256 channels: 16) share a tile.  They walk from barrier to barrier in step, so that matrix and vector
// unit are rarely busy at once: 1000 tokens over 32 groups of quant-groups of 64 with a cap took 472 us, where the folded form,
// whose waves pair up on several workgroups a compute unit, takes 286.  It is for the layouts that the folded form does not cover:
// 64 tokens over 128 groups of 196 in quant-groups of 16 134 us.
#pragma once

#include "oqm_attend_sums.h"

namespace oqm {

template <typename T, int DP_, bool BF16_META, int NW_, int MT_, bool SERIES>
struct Shared : Sums<T, DP_, (DP_ < 128 ? DP_ : 128), MT_, 1, SERIES> {
    typedef Sums<T, DP_, (DP_ < 128 ? DP_ : 128), MT_, 1, SERIES> S;
    typedef typename MetaPair<BF16_META>::type Pair;
    using S::GS, S::VU, S::STEPS, S::o;
    static constexpr int DP = DP_, MT = MT_, NW = NW_, THREADS = NW * 64;
    static constexpr int KP = kKeyParts<T>, PART = 32 * DP * 2, VALUES = KP * PART, STAGE = VALUES + 2 * PART;  // bytes in LDS
    // of a thread: key units (a token's 8 channels), value units (4 tokens' 2 channels)
    static constexpr int UNITS = 4 * DP, KU = (UNITS + THREADS - 1) / THREADS;

    struct Fetch {
        uint32_t k[KU][4], v[KU][4];  // rows: 8 channels, 4 x 2 channels; codes: the 32 bits that hold them
        Pair kp[KU], vp[KU][4];
        uint32_t k_shift[KU];         // how far up in them the codes of the keys stand
        bool stored, recent;
        uint32_t valid;               // of the tile's tokens
        int32_t t0, tokens;           // rows: first token, tokens of the segment
    };
    static __device__ __forceinline__ int32_t tiles(const AttendArgs& g) { return (g.k_eff * g.group_tokens + 31) / 32; }
    // Value unit i: two channels from c, tokens 16 * half + 4 * quarter + 0 .. 3.
    static __device__ __forceinline__ void value_unit(int i, int& c, int& half, int& quarter) {
        c = i % (DP / 2) * 2;
        half = i / (DP / 2) % 2;
        quarter = i / DP;
    }

    static __device__ __forceinline__ void fetch_rows(const AttendArgs& g, const AttendRows& r, int head, int32_t t0, int32_t tokens, Fetch& f) {
        const int tid = (int)threadIdx.x;
        f.stored = false;
        f.valid = 0xffffffffu;
        f.t0 = t0;
        f.tokens = tokens;
        const char* const k = r.k + head * r.k_head;
        const char* const v = r.v + head * r.v_head;
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int unit = i * THREADS + tid, c = unit / 32 % (DP / 8) * 8;
            const u32x4 x = *reinterpret_cast<const u32x4*>(k + (int64_t)min(t0 + unit % 32, tokens - 1) * r.k_row + (c < g.channels ? c : 0) * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) f.k[i][j] = x[j];
            f.k_shift[i] = 0;
            if constexpr (BF16_META && DP <= 128) f.kp[i] = 0;
        }
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            int c, half, quarter;
            value_unit((i * THREADS + tid) % UNITS, c, half, quarter);
            const char* const p = v + (c < g.channels ? c : 0) * 2;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f.v[i][j] = *reinterpret_cast<const uint32_t*>(p + (int64_t)min(t0 + 16 * half + 4 * quarter + j, tokens - 1) * r.v_row);
                if constexpr (BF16_META && DP <= 128) f.vp[i][j] = 0;  // all words of it on both sides, or some are kept in memory
            }
        }
    }
    // Where the tile's tokens stand.  In groups of 32 tokens or more they lie in two groups at most, and the slots are the wave's.
    struct Places {
        int64_t code[2], meta[2];  // of the two groups
        int32_t tok;               // the first token's row in its group
        bool there[2];
    };
    static __device__ __forceinline__ void fetch_stored(const AttendArgs& g, int head, int32_t t, Fetch& f) {
        const int tid = (int)threadIdx.x, lane = (int)__lane_id(), mine = lane & 31;
        f.stored = true;
        const int32_t tokens = g.k_eff * g.group_tokens;
        const char* const kc = g.codes[0] + head * g.code_head;
        const char* const vc = g.codes[1] + head * g.code_head;
        const Pair* const km = reinterpret_cast<const Pair*>(g.meta[0] + head * g.meta_head);
        const Pair* const vm = reinterpret_cast<const Pair*>(g.meta[1] + head * g.meta_head);
        const uint32_t row_bits = (uint32_t)g.channels * (uint32_t)g.bits;
        int32_t slot, tok;
        bool is;
        Places p;
        const bool two_groups = g.group_tokens >= 32;
        if (two_groups) {
            const int32_t rank = __builtin_amdgcn_readfirstlane((int)div_by((uint32_t)(t * 32), (uint32_t)g.group_tokens, g.inv_group_tokens));
            p.tok = t * 32 - rank * g.group_tokens;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int32_t s = -1;
                if (rank + i < g.k_eff) s = __builtin_amdgcn_readfirstlane(g.idx ? g.idx[rank + i] : rank + i);
                p.there[i] = s >= 0 && s < g.n_groups;
                if (!p.there[i]) s = 0;
                p.code[i] = s * g.code_slot;
                p.meta[i] = s * g.meta_slot;
            }
            tok = p.tok + mine;
            const bool second = tok >= g.group_tokens;
            if (second) tok -= g.group_tokens;
            is = (second ? p.there[1] : p.there[0]) && t * 32 + mine < tokens;
            slot = second;
        } else {
            const int32_t token = min(t * 32 + mine, tokens - 1);
            const uint32_t rank = div_by((uint32_t)token, (uint32_t)g.group_tokens, g.inv_group_tokens);
            tok = token - (int32_t)(rank * (uint32_t)g.group_tokens);
            const int32_t s = g.idx ? g.idx[rank] : (int32_t)rank;
            is = t * 32 + mine < tokens && s >= 0 && s < g.n_groups;
            slot = s >= 0 && s < g.n_groups ? s : 0;
        }
        f.valid = (uint32_t)__ballot(is);
        auto code_of = [&](int32_t s) { return two_groups ? (s ? p.code[1] : p.code[0]) : s * g.code_slot; };
        auto meta_of = [&](const Pair* base, int32_t s) {
            return reinterpret_cast<const Pair*>(reinterpret_cast<const char*>(base) + (two_groups ? (s ? p.meta[1] : p.meta[0]) : s * g.meta_slot));
        };
        const int64_t k_code = code_of(slot);
        const Pair* const k_meta = meta_of(km, slot);
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int c0 = (i * THREADS + tid) / 32 % (DP / 8) * 8, c = c0 < g.channels ? c0 : 0;
            const uint64_t at = reinterpret_cast<uint64_t>(kc) + (uint64_t)k_code + ((uint32_t)tok * row_bits + (uint32_t)(c * g.bits)) / 8;
            f.k[i][0] = *reinterpret_cast<const uint32_t*>(at & ~uint64_t{3});
            f.k[i][1] = f.k[i][2] = f.k[i][3] = 0;
            f.k_shift[i] = (uint32_t)(at & 3u) * 8u;
            f.kp[i] = k_meta[((uint32_t)tok * (uint32_t)g.channels + (uint32_t)c) >> g.qgroup_log2];
        }
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            int c0, half, quarter;
            value_unit((i * THREADS + tid) % UNITS, c0, half, quarter);
            const int c = c0 < g.channels ? c0 : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int from = 16 * half + 4 * quarter + j;  // the token, and a lane that has placed it
                int32_t v_slot, v_tok;
                if (two_groups) {
                    v_tok = p.tok + from;
                    v_slot = v_tok >= g.group_tokens;
                    if (v_slot) v_tok -= g.group_tokens;
                } else {
                    v_slot = __shfl(slot, from, 64);
                    v_tok = __shfl(tok, from, 64);
                }
                const uint32_t bits = (uint32_t)v_tok * row_bits + (uint32_t)(c * g.bits);
                f.v[i][j] = *reinterpret_cast<const uint8_t*>(vc + code_of(v_slot) + bits / 8);
                f.vp[i][j] = meta_of(vm, v_slot)[((uint32_t)v_tok * (uint32_t)g.channels + (uint32_t)c) >> g.qgroup_log2];
            }
        }
    }
    static __device__ __forceinline__ void put_values(char* at, const Operand<T>& hi, const Operand<T>& lo, bool two) {
        // the second channel's block lies 1 KB behind the first's
        *reinterpret_cast<u32x2*>(at) = u32x2{hi.w[0], hi.w[1]};
        *reinterpret_cast<u32x2*>(at + 1024) = u32x2{hi.w[2], hi.w[3]};
        if (two) {
            *reinterpret_cast<u32x2*>(at + PART) = u32x2{lo.w[0], lo.w[1]};
            *reinterpret_cast<u32x2*>(at + PART + 1024) = u32x2{lo.w[2], lo.w[3]};
        }
    }
    static __device__ __forceinline__ void stage(const AttendArgs& g, const Fetch& f, char* lds) {
        const int tid = (int)threadIdx.x;
        const uint32_t mask = g.bits == 4 ? 15u : 3u;
        const bool whole = f.valid == 0xffffffffu && g.channels == DP;  // nothing to be replaced by zero
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int unit = i * THREADS + tid, token = unit % 32, c8 = unit / 32;
            if (UNITS % THREADS != 0 && unit >= UNITS) break;
            char* const at = lds + ((token / 16 * STEPS + c8 % STEPS) * 64 + c8 / STEPS * 16 + token % 16) * 16;
            const bool inside = c8 * 8 < g.channels;
            if (f.stored) {
                f32x2 p = widen_pair(f.kp[i]);
                if (!whole && !((f.valid >> token & 1u) && inside)) p = f32x2{0.f, 0.f};
                const uint32_t w = f.k[i][0] >> f.k_shift[i];
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = __builtin_fmaf((float)(w >> (g.bits * j) & mask), p[0], p[1]);
                Operand<T> part[KP];
                split_key<T>(y, part);
#pragma unroll
                for (int j = 0; j < KP; ++j) *reinterpret_cast<u32x4*>(at + j * PART) = part[j].w;
            } else {
                *reinterpret_cast<u32x4*>(at) = inside ? u32x4{f.k[i][0], f.k[i][1], f.k[i][2], f.k[i][3]} : u32x4{0u, 0u, 0u, 0u};
            }
        }
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int unit = i * THREADS + tid;
            if (UNITS % THREADS != 0 && unit >= UNITS) break;
            int c, half, quarter;
            value_unit(unit, c, half, quarter);
            const int rest = c % GS, n = c / GS * VU + rest % VU, a = rest / VU;
            char* const at = lds + VALUES + ((n * 64 + quarter * 16 + a) * 8 + half * 4) * 2;
            Operand<T> hi, lo;
            if (f.stored) {
                const uint32_t there = c < g.channels ? f.valid >> (16 * half + 4 * quarter) : 0u, up = (uint32_t)(c * g.bits) & 7u;
                float y[8];  // channel c of the four tokens, then c + 1
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    f32x2 p = widen_pair(f.vp[i][j]);
                    if (!whole && !(there >> j & 1u)) p = f32x2{0.f, 0.f};
#pragma unroll
                    for (int u = 0; u < 2; ++u) y[4 * u + j] = __builtin_fmaf((float)(f.v[i][j] >> (up + (uint32_t)(g.bits * u)) & mask), p[0], p[1]);
                }
                split(y, hi, lo);
                put_values(at, hi, lo, true);
            } else {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = c < g.channels ? f.v[i][j] : 0u;
                hi.w = u32x4{__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u),
                             __builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
                put_values(at, hi, hi, false);
            }
        }
    }

    static __device__ __forceinline__ Operand<T> operand(const char* lds, int i) {
        Operand<T> x;
        x.w = *reinterpret_cast<const u32x4*>(lds + (i * 64 + (int)__lane_id()) * 16);
        return x;
    }
    // A staged tile.  two: it has more parts than one; valid: of its tokens; seen: of its tokens from the first, how many each query row sees.
    __device__ __forceinline__ void tile(const AttendArgs& g, const char* lds, const Operand<T> (&q)[MT][STEPS], bool two, uint32_t valid, const int32_t (&seen)[MT]) {
        const int quarter = (int)__lane_id() >> 4;
        f32x4 d[2][MT];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int m = 0; m < MT; ++m) d[half][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const Operand<T> x = operand(lds, half * STEPS + u);
#pragma unroll
                for (int m = 0; m < MT; ++m) d[half][m] = product(x, q[m][u], d[half][m]);
            }
        }
        if (two) {
#pragma unroll
            for (int i = 0; i < (KP - 1) * 2 * STEPS; ++i) {
                const int half = i / STEPS % 2, u = i % STEPS;
                const Operand<T> x = operand(lds + (1 + i / STEPS / 2) * PART, half * STEPS + u);
#pragma unroll
                for (int m = 0; m < MT; ++m) d[half][m] = product(x, q[m][u], d[half][m]);
            }
        }
        float w[MT][8], base[MT], start[MT];
        S::bases(g, base, start);
        bool all = valid == 0xffffffffu;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            all = all && seen[m] >= 32;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[m][i] = __builtin_fmaf(d[i / 4][m][i % 4], g.scale_log2, start[m]);
        }
        S::finish_scores(g, w, base);
        if (!__all(all)) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint32_t mine = (seen[m] >= 32 ? valid : seen[m] > 0 ? valid & ((1u << seen[m]) - 1u) : 0u) >> (4 * quarter);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!(mine >> (16 * (i / 4) + i % 4) & 1u)) w[m][i] = -__builtin_inff();
            }
        }
        this->probabilities(w, base);
        Operand<T> hi[MT], lo[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) split(w[m], hi[m], lo[m]);
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) {
            const Operand<T> x = operand(lds + VALUES, n);
#pragma unroll
            for (int m = 0; m < MT; ++m) o[m][n] = product(x, hi[m], o[m][n]);
#pragma unroll
            for (int m = 0; m < MT; ++m) o[m][n] = product(x, lo[m], o[m][n]);
        }
        if (two) {
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) {
                const Operand<T> x = operand(lds + VALUES + PART, n);
#pragma unroll
                for (int m = 0; m < MT; ++m) o[m][n] = product(x, hi[m], o[m][n]);
            }
        }
    }
};

template <typename F>
__global__ __launch_bounds__(F::THREADS, 2) void attend_shared_kernel(AttendArgs g) {
    typedef typename F::S S;
    typedef typename S::T T;
    constexpr int MT = F::MT, NW = F::NW, DP = F::DP, STEPS = S::STEPS, VU = S::VU, VN = S::VN, GS = S::GS;
    __shared__ __align__(16) char lds[2 * F::STAGE];
    const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
    const Item item = item_of(g, blockIdx.x);
    constexpr int kBlockRows = 16 * MT * NW;
    const int32_t rows = g.t_q * g.repeat;
    const int32_t first_row = (int32_t)item.block * kBlockRows, wave_row = first_row + wave * 16 * MT;

    F f;
    f.clear();
    bool there[MT];
    int32_t token[MT], q_head[MT];
    Operand<T> q[MT][STEPS];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int32_t row = wave_row + 16 * m + a;
        there[m] = row < rows;
        token[m] = there[m] ? (int32_t)div_by((uint32_t)row, (uint32_t)g.repeat, g.inv_repeat) : 0;
        q_head[m] = item.head * g.repeat + (there[m] ? row - token[m] * g.repeat : 0);
        const char* const p = g.q + q_head[m] * g.q_head + token[m] * g.q_row;
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int c = quarter * (DP / 4) + 8 * u;
            q[m][u].w = *reinterpret_cast<const u32x4*>(p + (c < g.channels ? c : 0) * 2);
            if (c >= g.channels) q[m][u].w = u32x4{0u, 0u, 0u, 0u};
        }
    }
    const bool works = wave_row < rows;  // a wave of a block's end has no rows but stages with the others
    const int32_t wave_last = (int32_t)div_by((uint32_t)(min(wave_row + 16 * MT, rows) - 1), (uint32_t)g.repeat, g.inv_repeat);
    const Segments s = segments_of(g, min(first_row + kBlockRows, rows) - 1, item.cut, 32, F::tiles(g));
    const int32_t stored_end = s.front_tiles + s.stored_tiles;

    typename F::Fetch next;
    auto fetch = [&](int32_t t) {
        next.recent = t >= stored_end;
        if (t < s.front_tiles) F::fetch_rows(g, g.front, item.head, t * 32, g.front.rows, next);
        else if (t < stored_end) F::fetch_stored(g, item.head, t - s.front_tiles, next);
        else F::fetch_rows(g, g.recent, item.head, (t - stored_end) * 32, s.recent_rows, next);
    };
    if (s.begin < s.end) {
        fetch(s.begin);
        F::stage(g, next, lds);
    }
    for (int32_t t = s.begin; t < s.end; ++t) {
        char* const here = lds + ((t - s.begin) & 1) * F::STAGE;
        char* const there_next = lds + ((t - s.begin + 1) & 1) * F::STAGE;
        const bool stored = next.stored, recent = next.recent;
        const uint32_t valid = next.valid;
        const int32_t t0 = next.t0, tokens = next.tokens;
        __syncthreads();  // the tile is there, and the other buffer has been read by all
        if (t + 1 < s.end) fetch(t + 1);
        if (works) {
            int32_t seen[MT];
            const bool causal = recent && g.causal;
            const int32_t all = stored ? 32 : (causal ? min(tokens, recent_seen(wave_last, g.recent.rows, g.t_q)) : tokens) - t0;
#pragma unroll
            for (int m = 0; m < MT; ++m) seen[m] = causal ? min(tokens, recent_seen(token[m], g.recent.rows, g.t_q)) - t0 : all;
            if (all > 0 && valid) f.tile(g, here, q, stored, valid, seen);
        }
        if (t + 1 < s.end) F::stage(g, next, there_next);
    }

#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float sum = f.sum[m];
        sum += lane_xor<16>(sum);
        sum += lane_xor<32>(sum);
        if (!there[m]) continue;
        typedef typename Element<T>::type E;
        const int64_t at = (int64_t)q_head[m] * g.t_q + token[m];
        const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int n = 0; n < VN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = n * GS + (4 * quarter + i) * VU;
                if (c >= g.channels) continue;
                if (g.splits > 1) {
                    typedef float Vec __attribute__((ext_vector_type(VU)));
                    Vec y;
#pragma unroll
                    for (int u = 0; u < VU; ++u) y[u] = f.o[m][n * VU + u][i];
                    *reinterpret_cast<Vec*>(g.part_out + (at * g.splits + item.cut) * g.channels + c) = y;
                } else {
                    typedef E Vec __attribute__((ext_vector_type(VU)));
                    Vec y;
#pragma unroll
                    for (int u = 0; u < VU; ++u) y[u] = (E)(f.o[m][n * VU + u][i] * by);
                    *reinterpret_cast<Vec*>(g.out + q_head[m] * g.out_head + token[m] * g.out_row + (int64_t)c * 2) = y;
                }
            }
        if (quarter == 0) {
            if (g.splits > 1) g.part_stat[at * g.splits + item.cut] = f32pair{f.ref[m], sum};
            else if (g.lse) g.lse[at] = sum > 0.0f ? (f.ref[m] + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
        }
    }
}

template <typename T, int DP, bool BF16_META>
void start_shared_of(const AttendArgs& g, hipStream_t s) {
    const dim3 grid((uint32_t)((int64_t)g.row_blocks * g.splits * g.kv_heads));
    constexpr int kMT = DP == 256 ? 1 : 2;
    if (g.cap_log2 > kPlainCap) launch(attend_shared_kernel<Shared<T, DP, BF16_META, 8, kMT, true>>, grid, dim3(512), 0, s, g);
    else launch(attend_shared_kernel<Shared<T, DP, BF16_META, 8, kMT, false>>, grid, dim3(512), 0, s, g);
}

template <typename T>
void start_shared(const AttendArgs& g, hipStream_t s) {
    if (g.meta_bf16) {
        if (g.channels <= 64) start_shared_of<T, 64, true>(g, s);
        else if (g.channels <= 128) start_shared_of<T, 128, true>(g, s);
        else start_shared_of<T, 256, true>(g, s);
    } else {
        if (g.channels <= 64) start_shared_of<T, 64, false>(g, s);
        else if (g.channels <= 128) start_shared_of<T, 128, false>(g, s);
        else start_shared_of<T, 256, false>(g, s);
    }
}

}  // namespace oqm
