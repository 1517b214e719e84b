// Rotary positions of new queries and keys, after a norm of every head where asked, and the copy of their values: one launch
// between a projection and the cache.
//
//   x' = x * w / sqrt(mean(x^2) + eps)                 (a, b) -> A (a cos t - b sin t, b cos t + a sin t), t = position * turns
//
// Every element is read once and written once, so memory bounds large calls and the launch small ones.  The cosines are the only
// arithmetic of weight: one float64 product and reduction a (token, pair), which the heads of a token share.
#include <cmath>

#include "oqm_attend.h"
#include "oqm_common.h"
#include "oqm_device.h"

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
template <typename T, int V, bool PAIRS, bool WIDE, bool PAST_CACHES>
__global__ __launch_bounds__(WIDE ? 1024 : kBlock) void rotate_kernel(RotateArgs g) {
    typedef typename Element<T>::type E;
    const uint32_t lanes = 1u << g.lanes_log2;
    const uint32_t slot = threadIdx.x & (lanes - 1);
    const uint64_t set = (uint64_t)blockIdx.x * (blockDim.x >> g.lanes_log2) + (threadIdx.x >> g.lanes_log2);
    if (set >= g.sets) return;  // whole sets: lanes of one leave together
    const uint32_t slow = div_by((uint32_t)set, g.fast, g.inv_fast), fast = (uint32_t)set - slow * g.fast;
    const uint32_t token = g.token_fast ? fast : slow, part = g.token_fast ? slow : fast;

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
        char* out = d.out + head * d.out_head + token * d.out_row;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (has[j]) store_elements<E, V, PAST_CACHES>(out + (int64_t)at[j] * sizeof(E), x[j]);
    }
}

template <typename T, int V, bool PAIRS>
void start_rotate_of(const RotateArgs& g, bool wide, bool large, dim3 grid, dim3 block, hipStream_t s) {
    if (wide) launch(rotate_kernel<T, V, PAIRS, true, false>, grid, block, 0, s, g);
    else if constexpr (V * elem_bytes<T>::value == 16) {
        if (large) launch(rotate_kernel<T, V, PAIRS, false, true>, grid, block, 0, s, g);
        else launch(rotate_kernel<T, V, PAIRS, false, false>, grid, block, 0, s, g);
    } else {
        launch(rotate_kernel<T, V, PAIRS, false, false>, grid, block, 0, s, g);
    }
}
template <typename T, int V>
void start_rotate(const RotateArgs& g, bool pairs, bool wide, bool large, dim3 grid, dim3 block, hipStream_t s) {
    if (pairs) start_rotate_of<T, V, true>(g, wide, large, grid, block, s);
    else start_rotate_of<T, V, false>(g, wide, large, grid, block, s);
}

static int bytes_of(int32_t dtype) { return dtype == TOM_F32 ? 4 : 2; }

static tom_status_t check_rotary(const tom_oqm_rotary_t* r) {
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

}  // namespace oqm

using namespace oqm;

extern "C" {

tom_status_t tom_oqm_rotary_turns(const tom_oqm_rotary_t* r, double* turns, float* amplitude) {
    if (tom_status_t st = check_rotary(r)) return st;
    if (!turns || !amplitude) return fail(TOM_ERR_INVALID_ARG, "turns and amplitude must be non-NULL");
    const double two_pi = 6.283185307179586476925;
    const int n = r->rotary_dim;
    const double base = r->scaling == TOM_ROTARY_BASE ? r->base * std::pow(r->factor, (double)n / (n - 2)) : r->base;
    double lo = 0, hi = 0;
    if (r->scaling == TOM_ROTARY_BY_PARTS) {
        // the pair that turns `times` times within the original length, as a real number
        auto place = [&](double times) { return n * std::log(r->original_length / (times * two_pi)) / (2 * std::log(base)); };
        lo = std::fmax(std::floor(place(32.0)), 0.0);
        hi = std::fmin(std::ceil(place(1.0)), n - 1.0);
    }
    for (int i = 0; i < n / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / n);
        double kept = 1.0;  // how much of the plain frequency stays
        if (r->scaling == TOM_ROTARY_LINEAR) kept = 0.0;
        if (r->scaling == TOM_ROTARY_BY_PARTS) kept = 1.0 - std::fmin(std::fmax((i - lo) / std::fmax(hi - lo, 0.001), 0.0), 1.0);
        if (r->scaling == TOM_ROTARY_BY_WAVELENGTH) kept = std::fmin(std::fmax((r->original_length * f / two_pi - 1.0) / 3.0, 0.0), 1.0);
        turns[i] = (f * kept + f / r->factor * (1.0 - kept)) / two_pi;
    }
    *amplitude = r->scaling == TOM_ROTARY_BY_PARTS ? (float)(0.1 * std::log(r->factor) + 1.0) : 1.0f;
    return TOM_OK;
}

tom_status_t tom_oqm_rotate(const tom_oqm_rotary_t* r, const double* turns, float amplitude, const int64_t* positions,
                            const tom_oqm_view_t* q, const tom_oqm_view_t* q_out, const tom_oqm_view_t* k, const tom_oqm_view_t* k_out,
                            const tom_oqm_view_t* v, const tom_oqm_view_t* v_out, const void* q_norm, const void* k_norm, float norm_eps,
                            void* hip_stream) {
    if (tom_status_t st = check_rotary(r)) return st;
    const tom_oqm_view_t* const in[3] = {q, k, v};
    const tom_oqm_view_t* const out[3] = {q_out, k_out, v_out};
    const void* const norm[3] = {q_norm, k_norm, nullptr};
    static const char* const name[3] = {"q", "k", "v"};
    const tom_oqm_view_t* one = nullptr;
    uintptr_t low_bits = 0;  // of every address and byte stride
    RotateArgs g{};
    constexpr int64_t kMaxStride = int64_t{1} << 40;  // elements; far beyond any device tensor
    for (int i = 0; i < 3; ++i) {
        if (!in[i] != !out[i]) return fail(TOM_ERR_INVALID_ARG, "%s and its output must both be given or both be NULL", name[i]);
        if (norm[i] && !in[i]) return fail(TOM_ERR_INVALID_ARG, "norm weights are given for %s, which is not", name[i]);
        if (!in[i]) continue;
        if (!one) one = in[i];
        for (const tom_oqm_view_t* t : {in[i], out[i]}) {
            if (t->dtype != TOM_F32 && t->dtype != TOM_BF16 && t->dtype != TOM_F16)
                return fail(TOM_ERR_INVALID_ARG, "the dtype of %s is not a tom_dtype_t", name[i]);
            if (t->dtype != one->dtype || t->rows != one->rows || t->channels != one->channels || t->heads != in[i]->heads)
                return fail(TOM_ERR_INVALID_ARG, "q, k, v and their outputs must agree in dtype, rows and channels, and each with its output in heads");
            if (t->heads < 0 || t->rows < 0) return fail(TOM_ERR_INVALID_ARG, "%s has a negative size", name[i]);
            if (t->head_stride < 0 || t->row_stride < 0 || t->head_stride > kMaxStride || t->row_stride > kMaxStride)
                return fail(TOM_ERR_INVALID_ARG, "strides of %s must be in [0, 2^40] elements", name[i]);
        }
        if (!elements_apart(*out[i])) return fail(TOM_ERR_INVALID_ARG, "heads or rows of %s's output overlap", name[i]);
    }
    if (!one) return TOM_OK;
    if (one->channels < r->rotary_dim || one->channels > 2048)
        return fail(TOM_ERR_INVALID_ARG, "channels = %d must be in [rotary_dim = %d, 2048]", one->channels, r->rotary_dim);
    if (!is_number(norm_eps) || norm_eps < 0.0f) return fail(TOM_ERR_INVALID_ARG, "norm_eps must be a number >= 0");
    if (!is_number(amplitude)) return fail(TOM_ERR_INVALID_ARG, "amplitude must be a number");
    int64_t heads = 0;
    for (int i = 0; i < 3; ++i)
        if (in[i]) heads += in[i]->heads;
    if (one->rows == 0 || heads == 0) return TOM_OK;
    const int e = bytes_of(one->dtype);
    for (int i = 0; i < 3; ++i) {
        RotateSide& d = g.side[i];
        if (!in[i] || in[i]->heads == 0) continue;
        if (!in[i]->data || !out[i]->data) return fail(TOM_ERR_INVALID_ARG, "%s and its output must have data", name[i]);
        d.in = static_cast<const char*>(in[i]->data);
        d.out = static_cast<char*>(out[i]->data);
        d.norm = static_cast<const char*>(norm[i]);
        // the stride of a size of one says nothing
        d.in_head = in[i]->heads > 1 ? in[i]->head_stride * e : 0;
        d.in_row = one->rows > 1 ? in[i]->row_stride * e : 0;
        d.out_head = in[i]->heads > 1 ? out[i]->head_stride * e : 0;
        d.out_row = one->rows > 1 ? out[i]->row_stride * e : 0;
        d.heads = in[i]->heads;
        d.turned = i < 2;
        low_bits |= reinterpret_cast<uintptr_t>(d.in) | reinterpret_cast<uintptr_t>(d.out) | reinterpret_cast<uintptr_t>(d.norm) |
                    (uintptr_t)d.in_head | (uintptr_t)d.in_row | (uintptr_t)d.out_head | (uintptr_t)d.out_row;
    }
    if (low_bits % e) return fail(TOM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    if (g.side[0].heads || g.side[1].heads) {
        if (!turns || !positions) return fail(TOM_ERR_INVALID_ARG, "turns and positions must be non-NULL");
        if ((reinterpret_cast<uintptr_t>(turns) | reinterpret_cast<uintptr_t>(positions)) & 7u)
            return fail(TOM_ERR_INVALID_ARG, "turns and positions must be 8-byte aligned");
    }
    if ((uint64_t)one->rows * (uint64_t)heads > 0x7fffffffu)
        return fail(TOM_ERR_UNSUPPORTED, "rows * heads exceeds 2^31 - 1: turn fewer rows per call");

    // Channels a lane moves at a time: as wide as the addresses and the shape of a head allow.
    const bool pairs = r->layout == TOM_ROTARY_PAIRS;
    int vec = 16 / e;
    while (vec > 1 && (low_bits % (uintptr_t)(vec * e) || (pairs ? r->rotary_dim % (2 * vec) : (r->rotary_dim / 2) % vec) || one->channels % vec)) vec /= 2;
    const int pair_slots = r->rotary_dim / (2 * vec);
    const int slots = pair_slots + (one->channels - r->rotary_dim + 2 * vec - 1) / (2 * vec);
    while ((1 << g.lanes_log2) < slots) ++g.lanes_log2;
    const uint32_t lanes = 1u << g.lanes_log2;
    const bool wide = lanes > 64;
    const uint32_t threads = wide ? lanes : kBlock;
    g.turns = turns;
    g.positions = positions;
    g.amplitude = amplitude;
    g.eps = norm_eps;
    g.inv_channels = 1.0f / (float)one->channels;
    g.rows = one->rows;
    g.channels = one->channels;
    g.rotary_dim = r->rotary_dim;
    g.pair_slots = pair_slots;
    g.heads = (uint32_t)heads;
    // Heads a lane takes one after the other share its cosines; small calls take one, so that every head has lanes of its own.  28 layers x
    // 4 heads x 12544 tokens of 128 channels (719 MB), us at 2 / 4 / 8 / 16 heads: 126.7 / 123.2 / 135.5 / 161.  28 + 2 * 4 heads of 128
    // channels, us of 300 / 700 / 1333 / 3000 / 6000 tokens: from 512K lanes up 7.46 / 7.73 / 7.64 / 11.97 / 20.16, never 7.37 /
    // 7.80 / 7.74 / 12.85 / 21.50, from 128K up 7.33 / 7.80 / 8.05 / 12.13 / 20.14.
    g.heads_per_lane = 1;
    while (g.heads_per_lane < 4 && (uint64_t)one->rows * heads * lanes / g.heads_per_lane > 512u * 1024u) g.heads_per_lane *= 2;
    g.parts = (g.heads + g.heads_per_lane - 1) / g.heads_per_lane;
    g.token_fast = one->row_stride < one->head_stride;
    g.fast = g.token_fast ? (uint32_t)one->rows : g.parts;
    g.inv_fast = reciprocal_u32(g.fast);
    g.sets = (uint64_t)g.parts * (uint64_t)one->rows;
    const uint32_t sets_per_block = threads / lanes;
    const uint64_t blocks = (g.sets + sets_per_block - 1) / sets_per_block;
    if (blocks * threads > kMaxLanes)
        return fail(TOM_ERR_UNSUPPORTED, "%d rows of %lld heads need more lanes than the 2^32 - 1 of a launch: turn fewer rows per call", one->rows, (long long)heads);
    const dim3 grid((uint32_t)blocks), block(threads);
    // Rows that the last-level cache (256 MB) cannot hold until somebody reads them are read and written past the caches.  The
    // same 719 MB, us, through / past: 138 / 123.2 = 5.8 TB/s.
    const bool large = (uint64_t)one->rows * (uint64_t)heads * (uint64_t)one->channels * (uint64_t)e * 2 >= (uint64_t)256 << 20;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
    if (e == 4) {
        if (vec == 4) start_rotate<In_f32, 4>(g, pairs, wide, large, grid, block, s);
        else if (vec == 2) start_rotate<In_f32, 2>(g, pairs, wide, large, grid, block, s);
        else start_rotate<In_f32, 1>(g, pairs, wide, large, grid, block, s);
    } else if (one->dtype == TOM_BF16) {
        if (vec == 8) start_rotate<In_bf16, 8>(g, pairs, wide, large, grid, block, s);
        else if (vec == 4) start_rotate<In_bf16, 4>(g, pairs, wide, large, grid, block, s);
        else if (vec == 2) start_rotate<In_bf16, 2>(g, pairs, wide, large, grid, block, s);
        else start_rotate<In_bf16, 1>(g, pairs, wide, large, grid, block, s);
    } else {
        if (vec == 8) start_rotate<In_f16, 8>(g, pairs, wide, large, grid, block, s);
        else if (vec == 4) start_rotate<In_f16, 4>(g, pairs, wide, large, grid, block, s);
        else if (vec == 2) start_rotate<In_f16, 2>(g, pairs, wide, large, grid, block, s);
        else start_rotate<In_f16, 1>(g, pairs, wide, large, grid, block, s);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(TOM_ERR_HIP, "rotate launch: %s", hipGetErrorString(err));
    return TOM_OK;
}

}  // extern "C"
