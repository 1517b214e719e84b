// Attention over pages for few query rows a sequence (one token, a short draft), and for float32.
//
// Memory bounds it: K and V are read once, straight into the operands of the matrix cores, no LDS and no barrier on the way.  S^T = K Q^T leaves a lane, for one
// query row, the scores of the very rows whose values it feeds to O^T = V^T P^T.  A workgroup has 16 query rows of a KV head; its four waves take the part's tiles
// of 32 rows in turn, each with sums of its own, and join them in LDS.  What hides memory's latency is the waves of a SIMD: as many as fit with no more than
// four vector registers spilled (1 or 2 in 16 bits of 128 channels, 2 or 3 in float32 of 64, 4 of 256; at 16 bits of 256 channels some 300 scalar ones, into lanes of vector registers).
//
// 28 query heads on 4 of 128 channels, bfloat16, both launches: 48 sequences of 40 to 30000 rows, a token each, 257 us (253 to 290 on different cards), 4.9 TB/s, where on the same card
// a copy reaches 4.98 and bare reads 6.76; one of 705 K rows 261 us (5.5 TB/s), of 12.6 K rows 13.1, of 500 rows 9.6, where the way from starts to table to rows to the join is what is left.
// Loads past the caches 337 us against 291.
#pragma once

#include "oqm_attend_pages_device.h"
#include "oqm_attend_sums.h"

namespace oqm {

template <typename T_, int DP_, bool SERIES>
struct PagedRows : Sums<T_, DP_, (DP_ < 128 ? DP_ : 128), 1, 1, SERIES> {
    typedef T_ T;
    typedef Sums<T_, DP_, (DP_ < 128 ? DP_ : 128), 1, 1, SERIES> S;
    using S::GS, S::VU, S::VN, S::STEPS, S::o;
    static constexpr int DP = DP_, E = elem_bytes<T>::value, KW = 8 * E / 16;  // KW: loads of 16 bytes of 8 channels
    static constexpr int WAVES = DP == 256 ? 1 : DP == 128 ? (E == 4 ? 2 : 3) : 4;                  // a SIMD: as many as their registers leave, see above
    static constexpr int VW = VU * E / 4;                                      // words of a value piece
    typedef uint32_t Piece __attribute__((ext_vector_type(VW)));
    bool sees_odd;

    // Channel c of what begins at p, or zeros where the head has no such channel.
    static __device__ __forceinline__ const char* channel(const PagesArgs& g, const char* p, int c) {
        return c < g.channels ? p + c * E : reinterpret_cast<const char*>(kZeroRow);
    }
    static __device__ __forceinline__ void load8(const char* p, Operand<T>& x) {
        if constexpr (E == 2) {
            x.w = *reinterpret_cast<const u32x4*>(p);
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) x.x[i] = a[i], x.x[4 + i] = b[i];
        }
    }
    // A tile of 32 rows; place: of row (lane & 31); there: the rows that are; see: of these the lane's query row's.
    __device__ __forceinline__ void tile(const PagesArgs& g, const char* k, const char* v, uint32_t place, const Operand<T> (&q)[1][STEPS], uint32_t there, uint32_t see) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        auto row = [&](const char* base, int i) {
            const uint32_t at = (uint32_t)__shfl((int)place, i, 64);
            return at == kNoPlace ? reinterpret_cast<const char*>(kZeroRow) : base + (int64_t)at * 16;
        };
        Operand<T> kx[2][STEPS];
        Piece vx[8][VN];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char* const p = row(k, 16 * half + a);
#pragma unroll
            for (int u = 0; u < STEPS; ++u) load8(channel(g, p, quarter * (DP / 4) + 8 * u), kx[half][u]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const char* const p = row(v, 16 * (i / 4) + 4 * quarter + i % 4);
#pragma unroll
            for (int n = 0; n < VN; ++n) vx[i][n] = *reinterpret_cast<const Piece*>(channel(g, p, n * GS + a * VU));
        }
        float w[1][8], base[1], start[1];
        S::bases(g, base, start);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < STEPS; ++u) d = product(kx[half][u], q[0][u], d);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[0][4 * half + i] = __builtin_fmaf(d[i], g.scale_log2, start[0]);
        }
        S::finish_scores(g, w, base);
        const uint32_t mine = see >> (4 * quarter);
        auto seen = [&](int i) { return (mine >> (16 * (i / 4) + i % 4) & 1u) != 0; };
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!seen(i)) w[0][i] = -__builtin_inff();
        this->probabilities(w, base);
        Operand<T> hi, lo;
        split(w[0], hi, lo);
        // Where a row is not for all, a probability of zero times what is not finite there would reach those who do not see it: such values become zero, and who sees such a
        // row is remembered.
        if (__any(see != there)) {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) odd = odd || odd_piece(vx[i]);
            if (__any(odd)) {
                uint32_t rows = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t lanes = __ballot(odd_piece(vx[i]));
#pragma unroll
                    for (int n = 0; n < 4; ++n) rows |= (uint32_t)(lanes >> (16 * n) & 0xffffu ? 1u : 0u) << (16 * (i / 4) + 4 * n + i % 4);
#pragma unroll
                    for (int n = 0; n < VN; ++n)
#pragma unroll
                        for (int u = 0; u < VW; ++u) vx[i][n][u] = without_odd<T>(vx[i][n][u]);
                }
                sees_odd = sees_odd || (rows & see) != 0;
            }
        }
#pragma unroll
        for (int n = 0; n < VN; ++n) {
            if constexpr (E == 2) {
#pragma unroll
                for (int u = 0; u < VU; u += 2) {
                    Operand<T> even, odd;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x = vx[2 * i][n][u / 2], y = vx[2 * i + 1][n][u / 2];
                        even.w[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                        odd.w[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                    }
                    f32x4 &e = o[0][n * VU + u], &f = o[0][n * VU + u + 1];
                    e = product(even, hi, e);
                    e = product(even, lo, e);
                    f = product(odd, hi, f);
                    f = product(odd, lo, f);
                }
            } else {
#pragma unroll
                for (int u = 0; u < VU; ++u) {
                    Operand<T> x;
#pragma unroll
                    for (int i = 0; i < 8; ++i) x.x[i] = __uint_as_float(vx[i][n][u]);
                    o[0][n * VU + u] = product(x, hi, o[0][n * VU + u]);
                }
            }
        }
    }
    static __device__ __forceinline__ bool odd_piece(const Piece (&x)[VN]) {
        bool odd = false;
#pragma unroll
        for (int n = 0; n < VN; ++n)
#pragma unroll
            for (int u = 0; u < VW; ++u) odd = odd || any_odd<T>(x[n][u]);
        return odd;
    }
};

constexpr int kPagedRows = 16, kPagedTile = 32;

template <typename F>
__global__ __launch_bounds__(kBlock, F::WAVES) void attend_pages_few_kernel(PagesArgs g) {
    typedef typename F::T T;
    constexpr int DP = F::DP, STEPS = F::STEPS, VU = F::VU, VN = F::VN, GS = F::GS, NW = kBlock / 64;
    __shared__ FoundItem found;
    __shared__ __align__(16) float sums[NW][kPagedRows][DP + 4];
    __shared__ f32pair stats[NW][kPagedRows];
    const uint32_t x = div_by(blockIdx.x, (uint32_t)g.kv_heads, g.inv_kv_heads);
    const int head = (int)(blockIdx.x - x * (uint32_t)g.kv_heads);
    Block b;
    if (!block_of<kPagedRows, kPagedTile, kBlock>(g, x, found, b)) return;
    const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
    tell_unit<kPagedRows>(g, b, x, head);

    const int32_t rows = b.tokens * g.repeat, row = b.tile * kPagedRows + a;
    const int32_t mine = row < rows ? row : rows - 1;
    const int32_t own = (int32_t)div_by((uint32_t)mine, (uint32_t)g.repeat, g.inv_repeat), token = b.first_token + own;
    const int32_t q_head = head * g.repeat + (mine - own * g.repeat);
    Operand<T> q[1][STEPS];
    {
        const char* const p = g.q + q_head * g.q_head + token * g.q_row;
#pragma unroll
        for (int u = 0; u < STEPS; ++u) F::load8(F::channel(g, p, quarter * (DP / 4) + 8 * u), q[0][u]);
    }
    const uint64_t* const mask = g.mask ? g.mask + (int64_t)token * g.words : nullptr;
    const int32_t* const table = g.p.table + (int64_t)b.sequence * g.p.table_pages;
    const char* const k = g.k + head * g.p.head_bytes;
    const char* const v = g.v + head * g.p.head_bytes;
    F f;
    f.clear();
    f.sees_odd = false;
    uint32_t next = kNoPlace;
    int32_t t0 = b.begin + wave * kPagedTile;
    if (t0 < b.end) next = place_of(g.p, table, (uint32_t)(t0 + (lane & 31)), (uint32_t)b.end);
    for (; t0 < b.end; t0 += NW * kPagedTile) {
        const uint32_t place = next;
        if (t0 + NW * kPagedTile < b.end) next = place_of(g.p, table, (uint32_t)(t0 + NW * kPagedTile + (lane & 31)), (uint32_t)b.end);
        const uint32_t there = (uint32_t)__ballot(place != kNoPlace);
        if (!there) continue;
        f.tile(g, k, v, place, q, there, there & (uint32_t)seen_from<kPagedTile>(g, t0, b.rows, own, mask));
    }
    float sum = f.sum[0];
    sum += lane_xor<16>(sum);
    sum += lane_xor<32>(sum);
    if (quarter == 0) stats[wave][a] = f32pair{f.ref[0], sum};
#pragma unroll
    for (int n = 0; n < VN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typedef float Vec __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int u = 0; u < VU; u += 4) {
                Vec y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = f.sees_odd ? __builtin_inff() : f.o[0][n * VU + u + j][i];
                *reinterpret_cast<Vec*>(&sums[wave][a][n * GS + (4 * quarter + i) * VU + u]) = y;
            }
        }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kPagedRows * DP / 4; i += kBlock) {
        const int r = i / (DP / 4), c = i % (DP / 4) * 4;
        const int32_t row_at = b.tile * kPagedRows + r;
        if (row_at >= rows || c >= g.channels) continue;
        float from = -__builtin_inff(), total = 0.0f;
        f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const f32pair st = stats[w][r];
            if (st.x == -__builtin_inff()) continue;
            const float top = fmaxf(from, st.x), old = exp2_of(from - top), new_ = exp2_of(st.x - top);
            from = top;
            total = total * old + st.y * new_;
            all = all * old + *reinterpret_cast<const f32x4*>(&sums[w][r][c]) * new_;
        }
        if (b.parts > 1) {
            const size_t slot = ((size_t)x * g.kv_heads + head) * kPagedRows + r;
            *reinterpret_cast<f32x4*>(g.part_out + slot * g.channels + c) = all;
            if (c == 0) g.part_stat[slot] = f32pair{from, total};
        } else {
            const int32_t t = (int32_t)div_by((uint32_t)row_at, (uint32_t)g.repeat, g.inv_repeat);
            const int32_t h = head * g.repeat + (row_at - t * g.repeat);
            const RowEnd end = row_end(g, h, b.first_token + t, from, total);
            put_channels<T>(g, h, b.first_token + t, c, all, end);
            if (c == 0) put_lse(g, h, b.first_token + t, end);
        }
    }
}

template <typename T, int DP>
void start_pages_few_of(const PagesArgs& g, hipStream_t s) {
    const dim3 grid(g.items * (uint32_t)g.kv_heads), block(kBlock);
    // (float32 takes the tanh by its series under any cap)
    if (g.cap_log2 > (__is_same(T, In_f32) ? 0.0f : kPlainCap)) launch(attend_pages_few_kernel<PagedRows<T, DP, true>>, grid, block, 0, s, g);
    else launch(attend_pages_few_kernel<PagedRows<T, DP, false>>, grid, block, 0, s, g);
}
template <typename T>
void start_pages_few(const PagesArgs& g, hipStream_t s) {
    if (g.channels <= 64) start_pages_few_of<T, 64>(g, s);
    else if (g.channels <= 128) start_pages_few_of<T, 128>(g, s);
    else start_pages_few_of<T, 256>(g, s);
    if (g.extra) start_join_pages<T, kPagedRows>(g, s);
}

}  // namespace oqm
