// Attention over pages for many query rows a sequence (drafts, prompts), in 16 bits.
//
// A workgroup has 32 query rows of a KV head for each of its NW waves, and its waves share staged tiles of KT rows, two in LDS: the next one is on its way (from
// memory into LDS past the registers) while a tile is worked on.  S^T = K Q^T in products of 32 x 32 x 16 leaves a lane, for one query row, the scores of 4 of
// each 8 rows; they become the operand of O^T = V^T P^T where they are, if V^T's rows are taken in the same order, which the transposing LDS read does.
// Probabilities enter as one part of the type, off by half a step of it each (2^-8 in bfloat16, 2^-11 in binary16): their error is no larger than that of the output's own
// rounding, and a second part would make the products of V twice as many.  Their sum is of the unrounded ones.
//
// In LDS a row lies as in memory, but its pieces of 16 bytes are exchanged by row, so that the lanes of a read, which differ in the row, do not meet in a bank.
//
// What bounds it.  28 query heads on 4, 128 channels: a prompt of 8192 tokens 472 to 502 us on different cards, 960 to 1020 TFLOP/s where a product of 8192^3 reaches 1180 to 1419.  With
// a part of the work left out: half of the products of K 134 us less, half of those of V 78, the staging 46, the exponentials 16, the reads of V 30, so it is the
// matrix cores first.  Three prompts of 1467 to 1994 tokens 348 to 363 us: their 560 workgroups do not divide evenly by 256 compute units.  4 drafts of 43 to 52
// tokens over 2000 to 7900 rows 35.3: 3 to find the part, 5.3 to the end of its first tile, 17.4 the others (16), 3.7 to write it, 7 to join; more tiles in LDS change nothing.
#pragma once

#include "oqm_attend_pages_device.h"
#include "oqm_attend_sums.h"

namespace oqm {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 product32(const Operand<In_bf16>& a, const Operand<In_bf16>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.w), __builtin_bit_cast(bf16x8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 product32(const Operand<In_f16>& a, const Operand<In_f16>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.w), __builtin_bit_cast(f16x8, b.w), c, 0, 0, 0);
}
// Four rows of 16 channels, 8 bytes a lane of 16, turned: lane i of 16 gets channel i of the four rows.
__device__ __forceinline__ u32x2 read_turned(const char* p) {
    typedef __attribute__((address_space(3))) s16x4* At;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(uint32_t)(uintptr_t)p));
}

// 16 bytes a lane from memory into LDS, lane after lane from `to`, past the registers.  Written out, since the compiler, which cannot tell what it overwrites, would
// wait for it in front of every turned read: the wait is wait_staged's.  (It has no register to write, and the address is taken when it is issued.)
__device__ __forceinline__ void load_to_lds(const char* p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(__builtin_amdgcn_readfirstlane(to)) : "m0", "memory");
}
__device__ __forceinline__ void wait_staged() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// tanh(y) / y by three terms where all of a wave's |y| are below a quarter (in units of z = 2 log2(e) y): four operations instead of two transcendental ones, a
// multiplication and an addition.  The terms are those whose largest relative error there is least, 2^-21.2 (found by exchange of its extrema).
constexpr float kSmallTanh = 0.25f * 2.0f * kLog2e;
constexpr float kTanh0 = 0.9999996043f, kTanh1 = -0.3332190823f, kTanh2 = 0.1284161343f;

// SPLIT: of 64 rows the first 32 are one half of the waves', the others the other half's, each with sums of its own that they join in LDS.
template <typename T_, int DP_, int NW_, bool SPLIT_, bool SERIES>
struct PagedTiles {
    typedef T_ T;
    static constexpr bool SPLIT = SPLIT_;
    static constexpr int DP = DP_, NW = NW_, KT = DP == 256 || NW < 4 ? 32 : 64, THREADS = NW * 64, QT = (SPLIT ? 16 : 32) * NW;
    static constexpr int ROW = DP * 2, CPR = ROW / 16, PART = KT * ROW, STAGE = 2 * PART;  // bytes; pieces of a row
    static constexpr int STEPS = DP / 16, NB = DP / 32;
    static constexpr int LOADS = KT * CPR / 64 / NW;  // of a wave, of K and of V
    static constexpr int WAVES = DP == 256 ? 1 : DP == 64 && NW < 8 ? 3 : 2;  // a SIMD, as many as their registers leave (two spilled at 128 channels and NW = 4; 64 channels of prompts, us, 2 / 3: 234 / 211)
    static constexpr int PLACES = NW == 8 ? 4096 : 1024;  // rows whose places are looked up at a time

    f32x16 o[NB];
    float ref, sum;

    static __device__ __forceinline__ int key_swap(int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int value_swap(int row) { return DP == 64 ? (row >> 1 & 1) << 2 : (row & 3) << 2; }

    // The tile's rows from memory into LDS, 16 bytes a lane, one behind the other; place: of row (lane % KT), any row's where there is none: what is not there is seen by
    // nobody, and channels that a head does not have meet zeros.
    static __device__ __forceinline__ void stage(const PagesArgs& g, const char* k, const char* v, uint32_t place, int wave, uint32_t lds) {
        const int lane = (int)__lane_id();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int first = (i * NW + wave) * 64, row = (first + lane) / CPR, piece = (first + lane) % CPR;
            const uint32_t at = (uint32_t)__shfl((int)place, row, 64);
            auto load = [&](const char* base, int c, uint32_t to) {
                if (c * 8 >= g.channels) c = 0;
                load_to_lds(base + c * 16 + (int64_t)at * 16, to);
            };
            load(k, piece ^ key_swap(row), lds + (uint32_t)(first * 16));
            load(v, piece ^ value_swap(row), lds + (uint32_t)(PART + first * 16));
        }
    }

    // The operand of V^T of channels 32 n .. 32 n + 31 and rows 16 t .. 16 t + 15 of a tile.
    static __device__ __forceinline__ Operand<T> values_of(const char* lds, int n, int t) {
        const int lane = (int)__lane_id(), i = lane & 15, side = lane >> 4 & 1, half = lane >> 5, row = 4 * half + i / 4;
        const char* const at = lds + (16 * t + row) * ROW + ((4 * n + 2 * side + i % 4 / 2) ^ value_swap(row)) * 16 + (i & 1) * 8;
        const u32x2 a = read_turned(at), b = read_turned(at + 8 * ROW);
        Operand<T> x;
        x.w = u32x4{a[0], a[1], b[0], b[1]};
        return x;
    }
    // Where a row is not for all, a probability of zero times what is not finite there would reach those who do not see it.  So rows with such values are looked for in those
    // tiles (every wave finds the same), and if there are any, the values become zero, and who sees such a row is remembered.
    static __device__ __forceinline__ uint64_t odd_rows(const char* lds) {
        auto odd_at = [&](int i) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(lds + PART + i * 16);
            return any_odd<T>(x[0]) || any_odd<T>(x[1]) || any_odd<T>(x[2]) || any_odd<T>(x[3]);
        };
        bool odd = false;
#pragma unroll 4
        for (int i = 0; i < KT * CPR; i += 64) odd = odd || odd_at(i + (int)__lane_id());
        if (!__any(odd)) return 0;
        odd = false;
#pragma unroll 1
        for (int i = 0; i < CPR; ++i) odd = odd || odd_at(((int)__lane_id() & (KT - 1)) * CPR + i);
        return __ballot(odd);
    }
    static __device__ __forceinline__ void clear_odd_values(char* lds) {
#pragma unroll 1
        for (int i = (int)threadIdx.x; i < KT * CPR; i += THREADS) {
            u32x4 x = *reinterpret_cast<const u32x4*>(lds + PART + i * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = without_odd<T>(x[j]);
            *reinterpret_cast<u32x4*>(lds + PART + i * 16) = x;
        }
    }

    // The operand of K of 32 rows and channels 16 u .. 16 u + 15.
    static __device__ __forceinline__ Operand<T> key_of(const char* lds, int u) {
        const int lane = (int)__lane_id(), half = lane >> 5, key = lane & 31;
        Operand<T> x;
        x.w = *reinterpret_cast<const u32x4*>(lds + key * ROW + ((2 * u + half) ^ key_swap(key)) * 16);
        return x;
    }
    static __device__ __forceinline__ void load_keys(const char* lds, Operand<T> (&x)[STEPS]) {
#pragma unroll
        for (int u = 0; u < STEPS; ++u) x[u] = key_of(lds, u);
    }
    // A staged tile.  there: its rows that are; see: of them the lane's query row's; part: whether that is to be asked at all.  Reads go out a phase ahead: the values' in
    // front of the softmax, the next keys' behind it, and the products find them there.
    __device__ __forceinline__ void tile(const PagesArgs& g, const char* lds, const Operand<T> (&q)[STEPS], bool part, uint64_t there, uint64_t see) {
        const int half = (int)__lane_id() >> 5;
        // (at 256 channels there are no registers for it)
        constexpr bool AHEAD = DP < 256;
        Operand<T> k[STEPS], v[NB][2];
        if constexpr (AHEAD) {
            load_keys(lds, k);
            __builtin_amdgcn_sched_barrier(0);
        }
        constexpr int BLOCKS = SPLIT ? 1 : KT / 32;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            if (b > 0 && !(uint32_t)(there >> 32)) return;
            const float base = ref == -__builtin_inff() ? 0.0f : ref;
            f32x16 d;
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = 0.0f;
#pragma unroll
            for (int u = 0; u < STEPS; ++u) d = product32(AHEAD ? k[u] : key_of(lds + 32 * b * ROW, u), q[u], d);
            if constexpr (AHEAD) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int t = 0; t < 2; ++t) v[n][t] = values_of(lds + PART, n, 2 * b + t);
                __builtin_amdgcn_sched_barrier(0);
            }
            // A bound of the scores' size, its own rounding counted in: of what is not seen too, and of negative ones, so that it only says when to look closer.
            float size = fabsf(d[0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) size = fmaxf(size, fabsf(d[i]));
            size *= fabsf(g.scale_log2) * (1.0f + 0x1p-20f);
            float w[16];
            if (g.cap_log2 == 0.0f) {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = __builtin_fmaf(d[i], g.scale_log2, -base);
            } else if (g.by_terms && !__any(size > kSmallTanh)) {
                // softcap tanh(y) = softcap y (k0 + k1 y^2 + k2 y^4), y = z / (2 log2 e)
                const float c0 = g.scale_log2 * g.cap_log2 * (0.5f * kLn2), y2 = g.scale_log2 * g.scale_log2 * (0.25f * kLn2 * kLn2);
                const float k0 = c0 * kTanh0, k1 = c0 * y2 * kTanh1, k2 = c0 * y2 * y2 * kTanh2;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = d[i] * d[i];
                    w[i] = __builtin_fmaf(d[i], __builtin_fmaf(x, __builtin_fmaf(x, k2, k1), k0), -base);
                }
            } else if constexpr (SERIES) {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = capped_exactly(d[i] * g.scale_log2, g.cap_log2) - base;
            } else {
                const float high = g.cap_log2 - base;
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = capped(d[i] * g.scale_log2, g.cap_log2, high);
            }
            if (part) {
                const uint32_t mine = (uint32_t)(see >> (32 * b + 4 * half));
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!(mine >> (8 * (i / 4) + i % 4) & 1u)) w[i] = -__builtin_inff();
            }
            const float level = (ref - base) + kRaised<T>;  // RAISED, or -infinity
            if (__any((g.cap_log2 != 0.0f ? g.cap_log2 * (0.5f * kLn2) * size : size) - base > level + kSlack<T>)) {
                float high = w[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) high = fmaxf(high, w[i]);
                if (__any(high > level + kSlack<T>)) {  // as in Sums::probabilities
                    high = fmaxf(high, lane_xor<32>(high));
                    const float peak = fmaxf(high, level);
                    const float by = exp2_of(fminf(kRaised<T> - peak, 0.0f)), down = fmaxf(peak, -__FLT_MAX__);
                    ref = base + (peak - kRaised<T>);
                    sum *= by;
#pragma unroll
                    for (int n = 0; n < NB; ++n) o[n] *= by;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        w[i] -= down;
                        if constexpr (kRaised<T> != 0.0f) w[i] += kRaised<T>;
                    }
                }
            }
            Operand<T> p[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    e[i] = exp2_of(w[8 * t + i]);
                    sum += e[i];
                }
                p[t].w = pack_items(T{}, e);
            }
            if constexpr (AHEAD) {
                if (b + 1 < BLOCKS) load_keys(lds + 32 * (b + 1) * ROW, k);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int t = 0; t < 2; ++t) o[n] = product32(AHEAD ? v[n][t] : values_of(lds + PART, n, 2 * b + t), p[t], o[n]);
        }
    }
};

template <typename F>
__global__ __launch_bounds__(F::THREADS, F::WAVES) void attend_pages_many_kernel(PagesArgs g) {
    typedef typename F::T T;
    constexpr int KT = F::KT, QT = F::QT, STEPS = F::STEPS, NB = F::NB;
    __shared__ FoundItem found;
    __shared__ __align__(16) char lds[2 * F::STAGE];
    __shared__ uint32_t places[F::PLACES];
    const uint32_t x = div_by(blockIdx.x, (uint32_t)g.kv_heads, g.inv_kv_heads);
    const int head = (int)(blockIdx.x - x * (uint32_t)g.kv_heads);
    Block b;
    if (!block_of<QT, KT, F::THREADS>(g, x, found, b)) return;
    tell_unit<QT>(g, b, x, head);
    const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    // Half of the waves go first, so that a SIMD's do not all want the matrix cores, and then the vector unit, at the same time.  Prompts of 1467 to 1994 tokens, us, without /
    // with: 64 channels 223 / 211, 128 and 256 the same; 4 drafts in halves of tiles 35.2 / 35.8.
    if (!F::SPLIT && wave >= F::NW / 2) __builtin_amdgcn_s_setprio(1);
    const int lane = (int)__lane_id(), half = lane >> 5;
    const int side = F::SPLIT ? wave / (F::NW / 2) : 0, row_wave = F::SPLIT ? wave % (F::NW / 2) : wave;

    const int32_t rows = b.tokens * g.repeat, row = b.tile * QT + row_wave * 32 + (lane & 31);
    const int32_t mine = row < rows ? row : rows - 1;
    const int32_t own = (int32_t)div_by((uint32_t)mine, (uint32_t)g.repeat, g.inv_repeat), token = b.first_token + own;
    const int32_t q_head = head * g.repeat + (mine - own * g.repeat);
    Operand<T> q[STEPS];
    {
        const char* const p = g.q + q_head * g.q_head + token * g.q_row;
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int c = 16 * u + 8 * half;
            q[u].w = *reinterpret_cast<const u32x4*>(c < g.channels ? p + c * 2 : reinterpret_cast<const char*>(kZeroRow));
        }
    }
    const uint64_t* const mask = g.mask ? g.mask + (int64_t)token * g.words : nullptr;
    const int32_t* const table = g.p.table + (int64_t)b.sequence * g.p.table_pages;
    const char* const k = g.k + head * g.p.head_bytes;
    const char* const v = g.v + head * g.p.head_bytes;
    const bool works = b.tile * QT + row_wave * 32 < rows;  // a wave of a block's end has no rows but stages with the others
    F f;
    f.ref = -__builtin_inff();
    f.sum = 0.0f;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) f.o[n][i] = 0.0f;

    constexpr uint64_t kAll = KT == 64 ? ~uint64_t{0} : 0xffffffffu;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    bool sees_odd = false;
    // the queries have arrived: waited for in the loop, they would be waited for in every round, and the staged rows with them
#pragma unroll
    for (int u = 0; u < STEPS; ++u) asm volatile("" : "+v"(q[u].w));
    auto entry = [&](int32_t r) { return table[div_by((uint32_t)min(r, b.end - 1), (uint32_t)g.p.page_rows, g.p.inv_page_rows)]; };
    auto place = [&](int32_t r, int32_t page) {  // of row r, whose entry that is
        if (r >= b.end || (uint32_t)page >= (uint32_t)g.p.n_pages) return kNoPlace;
        return (uint32_t)page * g.p.page_step + ((uint32_t)r - div_by((uint32_t)r, (uint32_t)g.p.page_rows, g.p.inv_page_rows) * (uint32_t)g.p.page_rows) * g.p.row_step;
    };
    auto stage = [&](uint32_t at, int buffer) {
        F::stage(g, k, v, at == kNoPlace ? 0u : at, wave, lds_at + (uint32_t)buffer * F::STAGE);
        return __ballot(at != kNoPlace) & kAll;
    };
    for (int32_t from = b.begin; from < b.end; from += F::PLACES) {
        const int32_t tiles = (min(b.end - from, F::PLACES) + KT - 1) / KT;
        if (from > b.begin) __syncthreads();  // the tiles and places before have been read
        // Places are looked up at once, not on the way (prompts of 1467 to 1994 tokens 380 us, 371 so); the first tile sets out with its
        // own entries, and they are written while it is on its way.
        constexpr int kFirst = 4;
        int32_t pages[kFirst];
#pragma unroll
        for (int u = 0; u < kFirst; ++u) pages[u] = entry(from + u * F::THREADS + (int32_t)threadIdx.x);
        uint64_t there = stage(place(from + lane % KT, entry(from + lane % KT)), 0);
#pragma unroll
        for (int u = 0; u < kFirst; ++u) {
            const int32_t i = u * F::THREADS + (int32_t)threadIdx.x;
            if (i < F::PLACES) places[i] = place(from + i, pages[u]);
        }
        for (int32_t i = kFirst * F::THREADS + (int32_t)threadIdx.x; i < tiles * KT; i += F::THREADS) places[i] = place(from + i, entry(from + i));
        for (int32_t n = 0; n < tiles; ++n) {
            const int32_t t0 = from + n * KT;
            char* const here = lds + (n & 1) * F::STAGE;
            wait_staged();
            __syncthreads();  // the tile is there (the places at first, too), and the other buffer has been read by all
            const uint64_t next = n + 1 < tiles ? stage(places[(n + 1) * KT + lane % KT], (n + 1) & 1) : 0;
            if (there) {
                const bool part = there != kAll || t0 + KT > b.for_all;
                uint64_t see = there;
                if (part) {
                    see &= seen_from<KT>(g, t0, b.rows, own, mask);
                    if (const uint64_t odd = F::odd_rows(here)) {
                        sees_odd = sees_odd || (odd & see) != 0;
                        __syncthreads();
                        F::clear_odd_values(here);
                        __syncthreads();
                    }
                }
                if (works && (uint32_t)(F::SPLIT ? there >> (32 * side) : 1u)) f.tile(g, here + side * 32 * F::ROW, q, part, there >> (32 * side), see >> (32 * side));
            }
            there = next;
        }
    }
    float sum = f.sum;
    sum += lane_xor<32>(sum);
    if constexpr (F::SPLIT) {
        __shared__ f32pair stats[QT];
        __shared__ bool odd[QT];
        f32x4* const sums = reinterpret_cast<f32x4*>(lds);
        __syncthreads();
        if (side == 1) {
#pragma unroll
            for (int i = 0; i < 4 * NB; ++i) sums[(row_wave * 4 * NB + i) * 64 + lane] = f32x4{f.o[i / 4][i % 4 * 4], f.o[i / 4][i % 4 * 4 + 1], f.o[i / 4][i % 4 * 4 + 2], f.o[i / 4][i % 4 * 4 + 3]};
            if (half == 0) {
                stats[row_wave * 32 + lane] = f32pair{f.ref, sum};
                odd[row_wave * 32 + lane] = sees_odd;
            }
        }
        __syncthreads();
        if (side == 1) return;
        const f32pair st = stats[row_wave * 32 + (lane & 31)];
        const float top = fmaxf(f.ref, st.x), from = top == -__builtin_inff() ? 0.0f : top;
        const float mine_by = exp2_of(f.ref - from), their_by = exp2_of(st.x - from);
        f.ref = top;
        sum = sum * mine_by + st.y * their_by;
        sees_odd = sees_odd || odd[row_wave * 32 + (lane & 31)];
#pragma unroll
        for (int i = 0; i < 4 * NB; ++i) {
            const f32x4 their = sums[(row_wave * 4 * NB + i) * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) f.o[i / 4][i % 4 * 4 + j] = f.o[i / 4][i % 4 * 4 + j] * mine_by + their[j] * their_by;
        }
    }
    if (row >= rows) return;
    if (sees_odd) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) f.o[n][i] = __builtin_inff();
    }
    if (b.parts > 1) {
        const size_t slot = ((size_t)x * g.kv_heads + head) * QT + row_wave * 32 + (lane & 31);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = 32 * n + 8 * j + 4 * half;
                if (c < g.channels) *reinterpret_cast<f32x4*>(g.part_out + slot * g.channels + c) = f32x4{f.o[n][4 * j], f.o[n][4 * j + 1], f.o[n][4 * j + 2], f.o[n][4 * j + 3]};
            }
        if (half == 0) g.part_stat[slot] = f32pair{f.ref, sum};
    } else {
        const RowEnd end = row_end(g, q_head, token, f.ref, sum);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = 32 * n + 8 * j + 4 * half;
                if (c < g.channels) put_channels<T>(g, q_head, token, c, f32x4{f.o[n][4 * j], f.o[n][4 * j + 1], f.o[n][4 * j + 2], f.o[n][4 * j + 3]}, end);
            }
        if (half == 0) put_lse(g, q_head, token, end);
    }
}

template <typename T, int DP, int NW, bool SPLIT>
void start_pages_many_of(const PagesArgs& g, hipStream_t s) {
    const dim3 grid(g.items * (uint32_t)g.kv_heads), block(64 * NW);
    if (g.cap_log2 > kPlainCap) launch(attend_pages_many_kernel<PagedTiles<T, DP, NW, SPLIT, true>>, grid, block, 0, s, g);
    else launch(attend_pages_many_kernel<PagedTiles<T, DP, NW, SPLIT, false>>, grid, block, 0, s, g);
    if (g.extra) start_join_pages<T, (SPLIT ? 16 : 32) * NW>(g, s);
}
template <typename T>
void start_pages_many(const PagesArgs& g, const PagesForm& form, hipStream_t s) {
    if (form.block_rows == 64) {
        if (g.channels <= 64) start_pages_many_of<T, 64, 2, false>(g, s);
        else if (g.channels <= 128) start_pages_many_of<T, 128, 2, false>(g, s);
        else start_pages_many_of<T, 256, 2, false>(g, s);
    } else if (form.block_rows == 128) {
        if (g.channels <= 64) {
            if (form.split) start_pages_many_of<T, 64, 8, true>(g, s);
            else start_pages_many_of<T, 64, 4, false>(g, s);
        } else if (g.channels <= 128) {
            if (form.split) start_pages_many_of<T, 128, 8, true>(g, s);
            else start_pages_many_of<T, 128, 4, false>(g, s);
        } else {
            start_pages_many_of<T, 256, 4, false>(g, s);
        }
    } else {
        start_pages_many_of<T, 128, 8, false>(g, s);
    }
}

}  // namespace oqm
