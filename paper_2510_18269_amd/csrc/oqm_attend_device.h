// What the kernels of the attention share: operands of the matrix cores, the two-part split, the cap, widened rows.
#pragma once

#include "oqm_attend.h"
#include "oqm_common.h"
#include "oqm_device.h"

namespace oqm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTile = 32;  // tokens

// The value of lane ^ N, without LDS.
template <int N>
__device__ __forceinline__ float lane_xor(float v) {
    static_assert(N == 8 || N == 16 || N == 32, "lane distance");
    if constexpr (N == 8) {
        return dpp_f32<0x128>(v);  // row_ror:8
    } else {
        // both registers hold v: the first ends with the lower lanes' (even rows') in all, the second with the others'
        uint32_t a = __float_as_uint(v), b = a;
        if constexpr (N == 32) swap32(a, b);
        else swap16(a, b);
        return __uint_as_float((__lane_id() & N) ? a : b);
    }
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// softcap * tanh(y) in units of log 2, from z = 2 log2(e) y: tanh y = 1 - 2 / (1 + 2^z).  The difference loses what the one has over
// tanh y: an error of 2^-22 * softcap at any y, which 16-bit results do not show up to a cap of 64 (2^-16).
// high: what z = infinity gives, cap_log2 or that less what scores are counted from.
__device__ __forceinline__ float capped(float z, float cap_log2, float high) {
    return __builtin_fmaf(-2.0f * cap_log2, __builtin_amdgcn_rcpf(1.0f + exp2_of(z)), high);
}
// Near zero by the series, for float32 and for caps above 64: there the error is 2^-22 of the score, and 2^-19 of it from an eighth of the cap on.
__device__ __forceinline__ float capped_exactly(float z, float cap_log2) {
    const float y = z * (0.5f * kLn2), x = y * y;
    const float small = y * fmaf(x, fmaf(x, fmaf(x, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    return x < 0.015625f ? cap_log2 * small : capped(z, cap_log2, cap_log2);
}

// ---- operands: 8 consecutive k of a row of a 16 x 16 x 32 product (16-bit types), or 8 products of one k a lane (float32) ----
template <typename T> struct Operand;
template <> struct Operand<In_bf16> {
    u32x4 w;
};
template <> struct Operand<In_f16> {
    u32x4 w;
};
template <> struct Operand<In_f32> {
    float x[8];
};
__device__ __forceinline__ f32x4 product(const Operand<In_bf16>& a, const Operand<In_bf16>& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w), __builtin_bit_cast(bf16x8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(const Operand<In_f16>& a, const Operand<In_f16>& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.w), __builtin_bit_cast(f16x8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(const Operand<In_f32>& a, const Operand<In_f32>& b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i], b.x[i], c, 0, 0, 0);
    return c;
}
// x = hi + lo + a rest of 2^-17 of it (bfloat16), or of 2^-23 of it but up to 2^-25 where it is small (binary16: half its last place there,
// no more than a reconstructed element loses when it is rounded to binary16); float32 has no rest in hi.
__device__ __forceinline__ void split(const float (&x)[8], Operand<In_bf16>& hi, Operand<In_bf16>& lo) {
    hi.w = pack_items(In_bf16{}, x);
    float r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[2 * i] = x[2 * i] - __uint_as_float(hi.w[i] << 16);
        r[2 * i + 1] = x[2 * i + 1] - __uint_as_float(hi.w[i] & 0xffff0000u);
    }
    lo.w = pack_items(In_bf16{}, r);
}
__device__ __forceinline__ void split(const float (&x)[8], Operand<In_f16>& hi, Operand<In_f16>& lo) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 v = {x[2 * i], x[2 * i + 1]};
        const f16x2 h = __builtin_convertvector(v, f16x2);  // v_cvt_pk_f16_f32
        // one instruction each, widening included
        const f32x2 r = {__builtin_fmaf((float)h[0], -1.0f, v[0]), __builtin_fmaf((float)h[1], -1.0f, v[1])};
        hi.w[i] = __builtin_bit_cast(uint32_t, h);
        lo.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(r, f16x2));
    }
}
__device__ __forceinline__ void split(const float (&x)[8], Operand<In_f32>& hi, Operand<In_f32>&) {
#pragma unroll
    for (int i = 0; i < 8; ++i) hi.x[i] = x[i];
}

// Keys that are reconstructed enter in as many parts as make them float32's: with outliers a score is a few hundred times the
// sum's last bits, and 2^-17 of it shows in the logarithm of the sum.
template <typename T> constexpr int kKeyParts = __is_same(T, In_f32) ? 1 : __is_same(T, In_f16) ? 2 : 3;
template <typename T>
__device__ __forceinline__ void split_key(const float (&x)[8], Operand<T> (&part)[kKeyParts<T>]) {
    if constexpr (kKeyParts<T> == 1) {
        Operand<T> none;
        split(x, part[0], none);
    } else if constexpr (kKeyParts<T> == 2) {
        split(x, part[0], part[1]);
    } else {
        Operand<T> ignored;
        split(x, part[0], ignored);
        float r[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r[2 * i] = x[2 * i] - __uint_as_float(part[0].w[i] << 16);
            r[2 * i + 1] = x[2 * i + 1] - __uint_as_float(part[0].w[i] & 0xffff0000u);
        }
        split(r, part[1], part[2]);
    }
}

// N (4 or 8) consecutive channels of a row in 32 bits.
template <typename T, int N>
__device__ __forceinline__ void load_row(const char* p, float* x) {
    if constexpr (N == 8) {
        Raw8<T> r;
        load_raw(p, r);
        float y[8];
        widen(r, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = y[i];
    } else if constexpr (elem_bytes<T>::value == 4) {
        const f32x4 r = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = r[i];
    } else {
        const u32x2 r = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint16_t h = (uint16_t)(r[i / 2] >> (16 * (i % 2)));
            if constexpr (__is_same(T, In_bf16)) x[i] = __uint_as_float((uint32_t)h << 16);
            else x[i] = (float)__builtin_bit_cast(_Float16, h);
        }
    }
}

// Codes and pairs of N (4 or 8) channels as they are in memory.  Branch-free whatever their widths, so that the loads of a tile are
// on their way together: codes are read as the aligned 32 bits that hold them (an array is a multiple of 4 bytes long), bfloat16
// pairs as the same 32 bits twice.
template <int N, bool TOKEN_AXIS>
struct Stored {
    static constexpr int NP = TOKEN_AXIS ? N : 1;
    uint32_t w, shift;
    __device__ __forceinline__ void load(const AttendArgs& g, const char* codes, uint32_t tok, int c) {
        const uint64_t at = reinterpret_cast<uint64_t>(codes) + ((uint64_t)tok * (uint32_t)g.channels + (uint32_t)c) * (uint32_t)g.bits / 8;
        w = *reinterpret_cast<const uint32_t*>(at & ~uint64_t{3});
        shift = (uint32_t)(at & 3u) * 8u;
    }
    __device__ __forceinline__ void values(const AttendArgs& g, const f32x2 (&pair)[NP], float* x) const {
        const uint32_t v = w >> shift, mask = g.bits == 4 ? 15u : 3u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const f32x2 p = pair[TOKEN_AXIS ? i : 0];
            x[i] = __builtin_fmaf((float)((v >> (g.bits * i)) & mask), p[0], p[1]);
        }
    }
};
struct StoredPair {
    uint32_t first, second;
    __device__ __forceinline__ void load(const AttendArgs& g, const char* meta, uint64_t i) {
        const char* p = meta + (g.meta_bf16 ? 4 : 8) * i;
        first = *reinterpret_cast<const uint32_t*>(p);
        second = *reinterpret_cast<const uint32_t*>(p + (g.meta_bf16 ? 0 : 4));
    }
    // of a token that is not there: zero, whatever has been read
    __device__ __forceinline__ f32x2 get(const AttendArgs& g, bool there) const {
        const uint32_t s = g.meta_bf16 ? first << 16 : first, m = g.meta_bf16 ? first & 0xffff0000u : second;
        return f32x2{__uint_as_float(there ? s : 0u), __uint_as_float(there ? m : 0u)};
    }
};

// Which block of query rows, part and KV head a number of the grid (or of a grid's waves) stands for.
struct Item {
    uint32_t block, cut;
    int head;
};
__device__ __forceinline__ Item item_of(const AttendArgs& g, uint32_t i) {
    const uint32_t rest = div_by(i, (uint32_t)g.row_blocks, g.inv_row_blocks), head = div_by(rest, (uint32_t)g.splits, g.inv_splits);
    return {i - rest * (uint32_t)g.row_blocks, rest - head * (uint32_t)g.splits, (int)head};
}

// Tiles of the three segments in one numbering, and what of them a part takes.
struct Segments {
    int32_t recent_rows, front_tiles, stored_tiles, begin, end;
};
__device__ __forceinline__ Segments segments_of(const AttendArgs& g, int32_t last_row, uint32_t cut, int tile_tokens, int32_t stored_tiles) {
    Segments s;
    s.recent_rows = g.recent.rows;  // as far as any row of the block sees
    if (g.causal) s.recent_rows = max(0, min(s.recent_rows, recent_seen((int32_t)div_by((uint32_t)last_row, (uint32_t)g.repeat, g.inv_repeat), g.recent.rows, g.t_q)));
    s.front_tiles = (g.front.rows + tile_tokens - 1) / tile_tokens;
    s.stored_tiles = stored_tiles;
    const uint32_t tiles = (uint32_t)(s.front_tiles + s.stored_tiles + (s.recent_rows + tile_tokens - 1) / tile_tokens);
    // equal runs, the first of them one longer where they do not divide evenly
    const uint32_t run = div_by(tiles, (uint32_t)g.splits, g.inv_splits), longer = tiles - run * (uint32_t)g.splits;
    s.begin = (int32_t)(cut * run + min(cut, longer));
    s.end = s.begin + (int32_t)run + (cut < longer ? 1 : 0);
    return s;
}

}  // namespace oqm
