// The kernel that turns rows to their positions, for outputs that are views and for rows of pages, and how a call is cut over the chip.
#pragma once

#include "oqm_pages.h"

namespace oqm {

struct RotateSide {  // queries, keys or values
    const char* in;
    char* out;
    const char* norm;  // weights [channels], or NULL
    int64_t in_head, in_row, out_head, out_row;  // bytes
    int32_t heads;     // 0: not given
    int32_t turned;
};
struct RotateArgs {
    RotateSide side[3];
    const double* turns;
    const int64_t* positions;
    float amplitude, eps, inv_channels;
    int32_t rows, channels, rotary_dim;
    int32_t pair_slots;       // lanes of a head that hold pairs; the following hold channels that do not turn
    uint32_t lanes_log2;      // lanes of a head
    uint32_t heads, heads_per_lane;   // of all sides; of them a lane takes this many, one after the other
    uint32_t parts, inv_fast, fast;   // parts of a token's heads; the faster of (part, token) in the numbering of the lane sets
    int32_t token_fast;
    uint64_t sets;
};
// Keys and values go to pages: side[1].out and side[2].out are those of the layer's first page, out_head is a head's step, out_row is not used.
struct AppendArgs : RotateArgs {
    PagePlaces pages;
};

template <typename E, int V>
struct Elements {  // as they are in memory: a load is not waited for until they are widened
    typedef E Vec __attribute__((ext_vector_type(V)));
    Vec r;
    template <bool PAST_CACHES>
    __device__ __forceinline__ void load(const char* p) {
        if constexpr (PAST_CACHES) r = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(p));
        else r = *reinterpret_cast<const Vec*>(p);
    }
    __device__ __forceinline__ void widen(float (&x)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)r[i];
    }
};
template <typename E, int V, bool PAST_CACHES>
__device__ __forceinline__ void store_elements(char* p, const float (&x)[V]) {
    typedef E Vec __attribute__((ext_vector_type(V)));
    Vec r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (E)x[i];
    if constexpr (PAST_CACHES) __builtin_nontemporal_store(r, reinterpret_cast<Vec*>(p));
    else *reinterpret_cast<Vec*>(p) = r;
}

// Cosine and sine of `turn` whole turns.  The nearest quarter turn is taken off in float64, exactly, and what remains, at most an
// eighth, rounded to float32; then the Taylor series of both (x = 2 pi r <= pi / 4: the terms left out are below 2^-28).  `turn` itself is a rounded
// product of float64: off by 2^-52 of the turns or so, which passes float32's last place of the cosine from position 10^9 on.
__device__ __forceinline__ void cos_sin_turns(double turn, float& c, float& s) {
    const double quarters = rint(turn * 4.0);
    const float r = (float)fma(quarters, -0.25, turn);
    const float z = r * r;
    // 2 pi, -(2 pi)^3 / 3!, ... and 1, -(2 pi)^2 / 2!, ...
    const float sn = r * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 42.058693944897653f, -76.705859753061386f), 81.605249276075054f), -41.341702240399755f), 6.283185307179586f);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -26.426256783374397f, 60.244641371876660f), -85.456817206693728f), 64.939394022668291f), -19.739208802178716f), 1.0f);
    // `quarters` modulo 4: beyond 2^31 it does not fit an int
    const int q = (int)(quarters - 4.0 * floor(quarters * 0.25));
    const float a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn;
    c = (q == 1 || q == 2) ? -a : a;
    s = (q >= 2) ? -b : b;
}

// A head is held by 2^lanes_log2 lanes of 2 V channels each: V pairs that turn (two runs of V channels half the rotary part
// apart, or one of 2 V), or 2 V channels behind them.  WIDE: more than a wave, and the sums of a norm are joined in LDS.
template <typename T, int V, bool PAIRS, bool WIDE, bool PAST_CACHES, typename ARGS>
__global__ __launch_bounds__(WIDE ? 1024 : kBlock) void rotate_kernel(ARGS g) {
    typedef typename Element<T>::type E;
    constexpr bool kPaged = __is_same(ARGS, AppendArgs);
    const uint32_t lanes = 1u << g.lanes_log2;
    const uint32_t slot = threadIdx.x & (lanes - 1);
    const uint64_t set = (uint64_t)blockIdx.x * (blockDim.x >> g.lanes_log2) + (threadIdx.x >> g.lanes_log2);
    if (set >= g.sets) return;  // whole sets: lanes of one leave together
    const uint32_t slow = div_by((uint32_t)set, g.fast, g.inv_fast), fast = (uint32_t)set - slow * g.fast;
    const uint32_t token = g.token_fast ? fast : slow, part = g.token_fast ? slow : fast;

    uint32_t place = 0;  // of the token's row
    if constexpr (kPaged) {
        const int32_t s = sequence_of(g.pages, (int32_t)token);
        if (s < 0) return;
        const int32_t begin = start_of(g.pages, s);
        const int64_t row = (int64_t)rows_of(g.pages, s) + ((int32_t)token - begin);
        place = kNoPlace;
        if (row < g.pages.capacity) place = place_of(g.pages, g.pages.table + (int64_t)s * g.pages.table_pages, (uint32_t)row, (uint32_t)g.pages.capacity);
    }
    const bool turns = (int)slot < g.pair_slots;
    int at[2];  // channels of the two runs
    if (turns) {
        at[0] = (int)slot * (PAIRS ? 2 * V : V);
        at[1] = PAIRS ? at[0] + V : at[0] + g.rotary_dim / 2;
    } else {
        at[0] = g.rotary_dim + ((int)slot - g.pair_slots) * 2 * V;
        at[1] = at[0] + V;
    }
    const bool has[2] = {at[0] < g.channels, at[1] < g.channels};

    const uint32_t first = part * g.heads_per_lane, last = min(first + g.heads_per_lane, g.heads);
    float cs[V], sn[V];
#pragma unroll
    for (int i = 0; i < V; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
    if (turns && first < (uint32_t)(g.side[0].heads + g.side[1].heads)) {
        const double position = (double)g.positions[token];
        const double* t = g.turns + (int)slot * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            cos_sin_turns(position * t[i], cs[i], sn[i]);
            cs[i] *= g.amplitude;
            sn[i] *= g.amplitude;
        }
    }

    for (uint32_t hh = first; hh < last; ++hh) {
        uint32_t w = 0, head = hh;
        if (head >= (uint32_t)g.side[0].heads) {
            head -= g.side[0].heads;
            w = 1;
            if (head >= (uint32_t)g.side[1].heads) {
                head -= g.side[1].heads;
                w = 2;
            }
        }
        const RotateSide d = w == 0 ? g.side[0] : w == 1 ? g.side[1] : g.side[2];  // selected: an index would be a load
        const char* in = d.in + head * d.in_head + token * d.in_row;
        Elements<E, V> raw[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (has[j]) raw[j].template load<PAST_CACHES>(in + (int64_t)at[j] * sizeof(E));
        float x[2][V];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) x[j][i] = 0.0f;
            if (has[j]) raw[j].widen(x[j]);
        }
        if (d.norm) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) sum = fmaf(x[j][i], x[j][i], sum);
            for (uint32_t m = min(lanes, 64u) / 2; m > 0; m /= 2) sum += __shfl_xor(sum, (int)m, 64);
            if constexpr (WIDE) {
                __shared__ float wave_sums[16];
                __syncthreads();  // the sums of the last head have been read
                if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = sum;
                __syncthreads();
                sum = 0.0f;
                for (uint32_t i = 0; i < lanes / 64; ++i) sum += wave_sums[i];
            }
            const float r = 1.0f / sqrtf(fmaf(sum, g.inv_channels, g.eps));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (!has[j]) continue;
                Elements<E, V> weight;
                weight.template load<false>(d.norm + (int64_t)at[j] * sizeof(E));
                float by[V];
                weight.widen(by);
#pragma unroll
                for (int i = 0; i < V; ++i) x[j][i] = x[j][i] * r * by[i];
            }
        }
        if (turns && d.turned) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float& a = PAIRS ? x[(2 * i) / V][(2 * i) % V] : x[0][i];
                float& b = PAIRS ? x[(2 * i + 1) / V][(2 * i + 1) % V] : x[1][i];
                const float p = a, q = b;
                a = p * cs[i] - q * sn[i];
                b = q * cs[i] + p * sn[i];
            }
        }
        char* out = d.out + head * d.out_head;
        if (kPaged && w > 0) {
            if (place == kNoPlace) continue;
            out += (int64_t)place * 16;
        } else {
            out += token * d.out_row;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (has[j]) store_elements<E, V, PAST_CACHES>(out + (int64_t)at[j] * sizeof(E), x[j]);
    }
}

template <typename T, int V, bool PAIRS, typename ARGS>
void start_rotate_of(const ARGS& g, bool wide, bool large, dim3 grid, dim3 block, hipStream_t s) {
    if (wide) launch(rotate_kernel<T, V, PAIRS, true, false, ARGS>, grid, block, 0, s, g);
    else if constexpr (V * elem_bytes<T>::value == 16) {
        if (large) launch(rotate_kernel<T, V, PAIRS, false, true, ARGS>, grid, block, 0, s, g);
        else launch(rotate_kernel<T, V, PAIRS, false, false, ARGS>, grid, block, 0, s, g);
    } else {
        launch(rotate_kernel<T, V, PAIRS, false, false, ARGS>, grid, block, 0, s, g);
    }
}
template <typename T, int V, typename ARGS>
void start_rotate(const ARGS& g, bool pairs, bool wide, bool large, dim3 grid, dim3 block, hipStream_t s) {
    if (pairs) start_rotate_of<T, V, true, ARGS>(g, wide, large, grid, block, s);
    else start_rotate_of<T, V, false, ARGS>(g, wide, large, grid, block, s);
}

inline tom_status_t check_rotary(const tom_oqm_rotary_t* r) {
    if (!r) return fail(TOM_ERR_INVALID_ARG, "rotary is NULL");
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > 2048)
        return fail(TOM_ERR_INVALID_ARG, "rotary_dim %d must be even, in [2, 2048]", r->rotary_dim);
    if (r->layout != TOM_ROTARY_HALF && r->layout != TOM_ROTARY_PAIRS) return fail(TOM_ERR_INVALID_ARG, "layout is not a tom_rotary_layout_t");
    if (r->scaling < TOM_ROTARY_PLAIN || r->scaling > TOM_ROTARY_BY_WAVELENGTH)
        return fail(TOM_ERR_INVALID_ARG, "scaling is not a tom_rotary_scaling_t");
    if (r->original_length < 1) return fail(TOM_ERR_INVALID_ARG, "original_length must be >= 1");
    if (!is_number(r->base) || r->base <= 1.0 || r->base > 1e30) return fail(TOM_ERR_INVALID_ARG, "base must be in (1, 1e30]");
    if (!is_number(r->factor) || r->factor < 1.0 || r->factor > 1e6) return fail(TOM_ERR_INVALID_ARG, "factor must be in [1, 1e6]");
    if (r->scaling == TOM_ROTARY_BASE && r->rotary_dim < 4) return fail(TOM_ERR_INVALID_ARG, "TOM_ROTARY_BASE needs a rotary_dim of 4 or more");
    return TOM_OK;
}

// Cuts the call over the chip and launches it.  The sides, positions, turns and (appended) pages of `g` are there; low_bits: of every address and
// byte stride; heads: of all sides, rows * heads below 2^31.
template <typename ARGS>
tom_status_t launch_rotate(ARGS& g, const tom_oqm_rotary_t* r, const char* what, int32_t dtype, int32_t rows, int32_t channels, int64_t heads, uintptr_t low_bits,
                           bool token_fast, float amplitude, float norm_eps, const double* turns, const int64_t* positions, void* hip_stream) {
    const int e = bytes_of_dtype(dtype);
    // Channels a lane moves at a time: as wide as the addresses and the shape of a head allow.
    const bool pairs = r->layout == TOM_ROTARY_PAIRS;
    int vec = 16 / e;
    while (vec > 1 && (low_bits % (uintptr_t)(vec * e) || (pairs ? r->rotary_dim % (2 * vec) : (r->rotary_dim / 2) % vec) || channels % vec)) vec /= 2;
    const int pair_slots = r->rotary_dim / (2 * vec);
    const int slots = pair_slots + (channels - r->rotary_dim + 2 * vec - 1) / (2 * vec);
    while ((1 << g.lanes_log2) < slots) ++g.lanes_log2;
    const uint32_t lanes = 1u << g.lanes_log2;
    const bool wide = lanes > 64;
    const uint32_t threads = wide ? lanes : kBlock;
    g.turns = turns;
    g.positions = positions;
    g.amplitude = amplitude;
    g.eps = norm_eps;
    g.inv_channels = 1.0f / (float)channels;
    g.rows = rows;
    g.channels = channels;
    g.rotary_dim = r->rotary_dim;
    g.pair_slots = pair_slots;
    g.heads = (uint32_t)heads;
    // Heads a lane takes one after the other share its cosines; small calls take one, so that every head has lanes of its own.  28 layers x
    // 4 heads x 12544 tokens of 128 channels (719 MB), us at 2 / 4 / 8 / 16 heads: 126.7 / 123.2 / 135.5 / 161.  28 + 2 * 4 heads of 128
    // channels, us of 300 / 700 / 1333 / 3000 / 6000 tokens: from 512K lanes up 7.46 / 7.73 / 7.64 / 11.97 / 20.16, never 7.37 /
    // 7.80 / 7.74 / 12.85 / 21.50, from 128K up 7.33 / 7.80 / 8.05 / 12.13 / 20.14.
    g.heads_per_lane = 1;
    while (g.heads_per_lane < 4 && (uint64_t)rows * heads * lanes / g.heads_per_lane > 512u * 1024u) g.heads_per_lane *= 2;
    g.parts = (g.heads + g.heads_per_lane - 1) / g.heads_per_lane;
    g.token_fast = token_fast;
    g.fast = g.token_fast ? (uint32_t)rows : g.parts;
    g.inv_fast = reciprocal_u32(g.fast);
    g.sets = (uint64_t)g.parts * (uint64_t)rows;
    const uint32_t sets_per_block = threads / lanes;
    const uint64_t blocks = (g.sets + sets_per_block - 1) / sets_per_block;
    if (blocks * threads > kMaxLanes)
        return fail(TOM_ERR_UNSUPPORTED, "%d rows of %lld heads need more lanes than the 2^32 - 1 of a launch: turn fewer rows per call", rows, (long long)heads);
    const dim3 grid((uint32_t)blocks), block(threads);
    // Rows that the last-level cache (256 MB) cannot hold until somebody reads them are read and written past the caches.  The
    // same 719 MB, us, through / past: 138 / 123.2 = 5.8 TB/s.
    const bool large = (uint64_t)rows * (uint64_t)heads * (uint64_t)channels * (uint64_t)e * 2 >= (uint64_t)256 << 20;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
    if (e == 4) {
        if (vec == 4) start_rotate<In_f32, 4, ARGS>(g, pairs, wide, large, grid, block, s);
        else if (vec == 2) start_rotate<In_f32, 2, ARGS>(g, pairs, wide, large, grid, block, s);
        else start_rotate<In_f32, 1, ARGS>(g, pairs, wide, large, grid, block, s);
    } else if (dtype == TOM_BF16) {
        if (vec == 8) start_rotate<In_bf16, 8, ARGS>(g, pairs, wide, large, grid, block, s);
        else if (vec == 4) start_rotate<In_bf16, 4, ARGS>(g, pairs, wide, large, grid, block, s);
        else if (vec == 2) start_rotate<In_bf16, 2, ARGS>(g, pairs, wide, large, grid, block, s);
        else start_rotate<In_bf16, 1, ARGS>(g, pairs, wide, large, grid, block, s);
    } else {
        if (vec == 8) start_rotate<In_f16, 8, ARGS>(g, pairs, wide, large, grid, block, s);
        else if (vec == 4) start_rotate<In_f16, 4, ARGS>(g, pairs, wide, large, grid, block, s);
        else if (vec == 2) start_rotate<In_f16, 2, ARGS>(g, pairs, wide, large, grid, block, s);
        else start_rotate<In_f16, 1, ARGS>(g, pairs, wide, large, grid, block, s);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(TOM_ERR_HIP, "%s launch: %s", what, hipGetErrorString(err));
    return TOM_OK;
}

}  // namespace oqm
