// Attention of new tokens over rows in front, stored groups as they are stored, and recent rows, in one softmax.
//
//   w_j = scale <q, k_j> (or softcap tanh of it / softcap)      out = sum_j exp(w_j - M) v_j / sum_j exp(w_j - M)
//
// One pass over the keys and values with the running maximum and sum of each query row.  The keys' product is taken transposed,
// S^T = K Q^T on the matrix cores: a lane then holds, for one query row, the scores of the very tokens whose values it feeds as
// the other operand of O^T = V^T P^T, so that the probabilities never leave their lane.
#include "oqm_attend_device.h"

namespace oqm {

// ---- general form ------------------------------------------------------------------------------------------------------------
// A wave takes 16 query rows of a KV head and a run of 32-token tiles, on its own: every element is reconstructed (or widened) to
// float32 and enters the products in two 16-bit parts where one does not hold it.  DP: channels, padded with zeros.
//   K operand  lane (token l % 16 of a half, quarter l / 16): DP / 4 consecutive channels
//   V operand  lane (l % 16, l / 16): of the 8 tokens whose scores it holds, VN runs of VU channels
// Along the tokens' axis a tile lies in one group, whose pairs a lane then reads once.  Where a tile's channels are padding or a
// token is not there, what is read instead is some valid place, and not used.
// Latency bounds it where rows are few (float32, 2 heads of 64 channels, 72 rows: 7 us), the vector unit, which takes every
// element apart in every wave, where they are many: 36 bfloat16 tokens of 28 heads over 64 groups of 50 in quant-groups of 16 53 us.
template <typename T, int DP, bool TOKEN_AXIS>
struct General {
    static constexpr int VU = DP / 16 < 8 ? DP / 16 : 8, VN = DP / 16 / VU, STEPS = DP / 32;
    static constexpr bool EARLY = DP * elem_bytes<T>::value <= 256;  // the values' loads go out with the keys': there are registers for both
    static constexpr bool LATE_PAIRS = TOKEN_AXIS && DP > 64;        // for so many pairs there are not
    // A dot in float32 is added up in as many chains, joined by pairs: results of 256 channels with outlier keys 2.4e-6 from 64 bits with
    // one chain, 1.2e-6 with four.
    static constexpr int CHAINS = !__is_same(T, In_f32) ? 1 : STEPS < 4 ? STEPS : 4;
    // Probabilities of binary16 are raised by 2^15 until the sums are done: two parts of one end at 2^-25, and so would the tail of a softmax.
    static constexpr float RAISED = __is_same(T, In_f16) ? 15.0f : 0.0f;
    Operand<T> q[STEPS];
    f32x4 o[DP / 16];
    float top, sum;

    static __device__ __forceinline__ void join_chains(f32x4 (&s)[2][CHAINS]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if constexpr (CHAINS == 2) s[half][0] += s[half][1];
            if constexpr (CHAINS == 4) s[half][0] = (s[half][0] + s[half][1]) + (s[half][2] + s[half][3]);
        }
    }
    static __device__ __forceinline__ int32_t tiles(const AttendArgs& g) {
        if constexpr (TOKEN_AXIS) return g.k_eff * ((g.group_tokens + kTile - 1) / kTile);
        return (g.k_eff * g.group_tokens + kTile - 1) / kTile;
    }

    __device__ __forceinline__ void softmax(const AttendArgs& g, float (&w)[8]) {
        float high = w[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) high = fmaxf(high, w[i]);
        if (__any(high > top)) {
            high = fmaxf(high, lane_xor<16>(high));
            high = fmaxf(high, lane_xor<32>(high));
            const float next = fmaxf(top, high);
            const float by = next == -__builtin_inff() ? 1.0f : exp2_of((top - next) * g.score_unit);
            top = next;
            sum *= by;
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) o[n] *= by;
        }
        const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (RAISED != 0.0f) w[i] = exp2_of(__builtin_fmaf(w[i] - from, g.score_unit, RAISED));
            else w[i] = exp2_of((w[i] - from) * g.score_unit);
            sum += w[i];
        }
    }
    __device__ __forceinline__ float score(const AttendArgs& g, float dot, bool seen) const {
        const float y = dot * g.scale_log2;
        const float z = g.cap_log2 != 0.0f ? capped_exactly(y, g.cap_log2) : y;
        return seen ? z : -__builtin_inff();
    }
    // One block of the sums: values of the lane's 8 tokens in one channel.
    template <bool EXACT>
    __device__ __forceinline__ void add(f32x4& acc, const float (&y)[8], const Operand<T>& ph, const Operand<T>& pl) {
        Operand<T> hi, lo;
        split(y, hi, lo);
        acc = product(hi, ph, acc);
        if constexpr (!__is_same(T, In_f32)) {
            acc = product(hi, pl, acc);
            if constexpr (!EXACT) acc = product(lo, ph, acc);
        }
    }

    __device__ __forceinline__ void stored(const AttendArgs& g, int head, int32_t t) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        const char* const kc = g.codes[0] + head * g.code_head;
        const char* const vc = g.codes[1] + head * g.code_head;
        const char* const km = g.meta[0] + head * g.meta_head;
        const char* const vm = g.meta[1] + head * g.meta_head;
        // the tile's 32 tokens, one of each half a lane
        int32_t slot[2], tok[2];
        bool is[2];
        if constexpr (TOKEN_AXIS) {
            const int32_t parts = (g.group_tokens + kTile - 1) / kTile, rank = t / parts, first = (t - rank * parts) * kTile;
            const int32_t s = g.idx ? g.idx[rank] : rank;
            const bool there = s >= 0 && s < g.n_groups;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                slot[half] = there ? s : 0;
                is[half] = there && first + 16 * half + a < g.group_tokens;
                tok[half] = min(first + 16 * half + a, g.group_tokens - 1);
            }
        } else {
            const int32_t tokens = g.k_eff * g.group_tokens;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int32_t token = min(t * kTile + 16 * half + a, tokens - 1);
                const uint32_t rank = div_by((uint32_t)token, (uint32_t)g.group_tokens, g.inv_group_tokens);
                tok[half] = token - (int32_t)(rank * (uint32_t)g.group_tokens);
                const int32_t s = g.idx ? g.idx[rank] : (int32_t)rank;
                is[half] = t * kTile + 16 * half + a < tokens && s >= 0 && s < g.n_groups;
                slot[half] = s >= 0 && s < g.n_groups ? s : 0;
            }
        }
        typedef Stored<8, TOKEN_AXIS> Key;
        typedef Stored<VU, TOKEN_AXIS> Value;
        Key kx[2][STEPS];
        StoredPair kp[TOKEN_AXIS ? 1 : 2][LATE_PAIRS ? 1 : STEPS][Key::NP];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int c = quarter * (DP / 4) + 8 * u, at = c < g.channels ? c : 0;
                kx[half][u].load(g, kc + slot[half] * g.code_slot, (uint32_t)tok[half], at);
                if constexpr (TOKEN_AXIS) {
                    if (half == 0 && !LATE_PAIRS)
#pragma unroll
                        for (int i = 0; i < 8; ++i) kp[0][LATE_PAIRS ? 0 : u][i].load(g, km + slot[0] * g.meta_slot, (uint64_t)(at + i));
                } else {
                    kp[half][u][0].load(g, km + slot[half] * g.meta_slot, ((uint64_t)(uint32_t)tok[half] * (uint32_t)g.channels + (uint32_t)at) >> g.qgroup_log2);
                }
            }
        // slots and rows of the tokens whose scores the lane holds
        int32_t v_slot[8], v_tok[8];
        uint32_t v_is = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v_slot[j] = __shfl(slot[j / 4], 4 * quarter + j % 4, 64);
            v_tok[j] = __shfl(tok[j / 4], 4 * quarter + j % 4, 64);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) v_is |= (uint32_t)((__ballot(is[half]) >> (4 * quarter)) & 15u) << (4 * half);
        Value vx[VN][8];
        StoredPair vp[VN][TOKEN_AXIS ? 1 : 8][Value::NP];
        auto load_values = [&] {
#pragma unroll
            for (int v = 0; v < VN; ++v) {
                const int c = v * 16 * VU + a * VU, at = c < g.channels ? c : 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    vx[v][j].load(g, vc + v_slot[j] * g.code_slot, (uint32_t)v_tok[j], at);
                    if constexpr (TOKEN_AXIS) {
                        if (j == 0)
#pragma unroll
                            for (int i = 0; i < VU; ++i) vp[v][0][i].load(g, vm + v_slot[0] * g.meta_slot, (uint64_t)(at + i));
                    } else {
                        vp[v][j][0].load(g, vm + v_slot[j] * g.meta_slot, ((uint64_t)(uint32_t)v_tok[j] * (uint32_t)g.channels + (uint32_t)at) >> g.qgroup_log2);
                    }
                }
            }
        };
        if constexpr (EARLY) load_values();
        float w[8];
        f32x4 s[2][CHAINS];
#pragma unroll
        for (int i = 0; i < 2 * CHAINS; ++i) s[i / CHAINS][i % CHAINS] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int c = quarter * (DP / 4) + 8 * u;
            const bool inside = c < g.channels;
            if constexpr (LATE_PAIRS) {
                asm volatile("" ::: "memory");  // not before they are wanted
#pragma unroll
                for (int i = 0; i < 8; ++i) kp[0][0][i].load(g, km + slot[0] * g.meta_slot, (uint64_t)((inside ? c : 0) + i));
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x2 pair[Key::NP];
#pragma unroll
                for (int i = 0; i < Key::NP; ++i) pair[i] = kp[TOKEN_AXIS ? 0 : half][LATE_PAIRS ? 0 : u][i].get(g, is[half] && inside);
                float x[8];
                kx[half][u].values(g, pair, x);
                Operand<T> part[kKeyParts<T>];
                split_key<T>(x, part);
                f32x4& d = s[half][u % CHAINS];
#pragma unroll
                for (int i = 0; i < kKeyParts<T>; ++i) d = product(part[i], q[u], d);
            }
        }
        join_chains(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = score(g, s[i / 4][0][i % 4], v_is >> i & 1u);
        softmax(g, w);
        if constexpr (!EARLY) load_values();
        Operand<T> ph, pl;
        split(w, ph, pl);
#pragma unroll
        for (int v = 0; v < VN; ++v) {
            float x[8][VU];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f32x2 pair[Value::NP];
#pragma unroll
                for (int i = 0; i < Value::NP; ++i) pair[i] = vp[v][TOKEN_AXIS ? 0 : j][i].get(g, v_is >> j & 1u);
                vx[v][j].values(g, pair, x[j]);
            }
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j][i];
                add<false>(o[v * VU + i], y, ph, pl);
            }
        }
    }

    // A tile of rows as the model has them, from t0; `seen`: of the rows from the first, how many the lane's query row sees.
    __device__ __forceinline__ void rows(const AttendArgs& g, const AttendRows& r, int head, int32_t t0, int32_t tokens, int32_t seen) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        const char* const k = r.k + head * r.k_head;
        const char* const v = r.v + head * r.v_head;
        constexpr int E = elem_bytes<T>::value;
        Raw8<T> kx[2][STEPS];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int c = quarter * (DP / 4) + 8 * u;
                load_raw(k + min(t0 + 16 * half + a, tokens - 1) * r.k_row + (int64_t)(c < g.channels ? c : 0) * E, kx[half][u]);
            }
        typedef uint32_t Run __attribute__((ext_vector_type(VU * E / 4)));
        Run vx[VN][8];
        auto load_values = [&] {
#pragma unroll
            for (int n = 0; n < VN; ++n)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = n * 16 * VU + a * VU;
                    const char* p = v + min(t0 + 16 * (j / 4) + 4 * quarter + j % 4, tokens - 1) * r.v_row + (int64_t)(c < g.channels ? c : 0) * E;
                    __builtin_memcpy(&vx[n][j], __builtin_assume_aligned(p, VU * E < 16 ? VU * E : 16), sizeof(Run));
                }
        };
        if constexpr (EARLY) load_values();
        float w[8];
        f32x4 s[2][CHAINS];
#pragma unroll
        for (int i = 0; i < 2 * CHAINS; ++i) s[i / CHAINS][i % CHAINS] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                float x[8];
                widen(kx[half][u], x);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = quarter * (DP / 4) + 8 * u < g.channels ? x[i] : 0.0f;
                Operand<T> hi, lo;
                split(x, hi, lo);
                s[half][u % CHAINS] = product(hi, q[u], s[half][u % CHAINS]);
            }
        join_chains(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = score(g, s[i / 4][0][i % 4], t0 + 16 * (i / 4) + 4 * quarter + i % 4 < seen);
        softmax(g, w);
        if constexpr (!EARLY) load_values();
        Operand<T> ph, pl;
        split(w, ph, pl);
#pragma unroll
        for (int n = 0; n < VN; ++n)
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (E == 4) y[j] = __uint_as_float(vx[n][j][i]);
                    else if constexpr (__is_same(T, In_bf16)) y[j] = __uint_as_float(i % 2 ? vx[n][j][i / 2] & 0xffff0000u : vx[n][j][i / 2] << 16);
                    else y[j] = (float)__builtin_bit_cast(_Float16, (uint16_t)(vx[n][j][i / 2] >> (16 * (i % 2))));
                }
                add<true>(o[n * VU + i], y, ph, pl);
            }
    }
};

// Waves a SIMD: 192 channels, 196 tokens a group, in quant-groups of 32, with one / two: 24 bfloat16 tokens over 64 groups 172 / 136 us,
// one over 1000 233 / 172; 64 float32 ones 480 / 382; 96 channels with two / three: 72.0 / 70.7, 88.7 / 88.9, 199 / 200.  Along the
// tokens, of groups of 50, whose pairs want the registers, with one / two: 97 / 145, 117 / 180, 247 / 389.
template <typename T, int DP, bool TOKEN_AXIS>
__global__ __launch_bounds__(kBlock, DP == 64 ? (TOKEN_AXIS ? 2 : 3) : DP == 128 || !TOKEN_AXIS ? 2 : 1) void attend_kernel(AttendArgs g) {
    typedef General<T, DP, TOKEN_AXIS> Form;
    const Item item = item_of(g, (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kBlock / 64) + threadIdx.x / 64)));
    const uint32_t cut = item.cut;
    const int head = item.head;
    if (head >= g.kv_heads) return;
    const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
    // query rows of a KV head: token-major, so that a block of them ends at about one token
    const int32_t rows = g.t_q * g.repeat;
    const int32_t row = (int32_t)item.block * 16 + a;
    const bool there = row < rows;
    const int32_t token = there ? (int32_t)div_by((uint32_t)row, (uint32_t)g.repeat, g.inv_repeat) : 0;
    const int32_t q_head = head * g.repeat + (there ? row - token * g.repeat : 0);

    Form f;
    f.top = -__builtin_inff();
    f.sum = 0.0f;
#pragma unroll
    for (int n = 0; n < DP / 16; ++n) f.o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    // A row that is not there computes with the first one, so that nothing waits for a condition.
    Raw8<T> raw[Form::STEPS];
    const char* const q_row = g.q + q_head * g.q_head + token * g.q_row;
#pragma unroll
    for (int u = 0; u < Form::STEPS; ++u) {
        const int c = quarter * (DP / 4) + 8 * u;
        load_raw(q_row + (int64_t)(c < g.channels ? c : 0) * elem_bytes<T>::value, raw[u]);
    }
#pragma unroll
    for (int u = 0; u < Form::STEPS; ++u) {
        float x[8];
        widen(raw[u], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = quarter * (DP / 4) + 8 * u < g.channels ? x[i] : 0.0f;
        Operand<T> unused;
        split(x, f.q[u], unused);
    }

    const Segments s = segments_of(g, min((int32_t)item.block * 16 + 15, rows - 1), cut, kTile, Form::tiles(g));
    const int32_t recent = s.recent_rows, stored_end = s.front_tiles + s.stored_tiles;
    const int32_t seen = !there ? 0 : g.causal ? min(recent, recent_seen(token, g.recent.rows, g.t_q)) : recent;
    for (int32_t t = s.begin; t < min(s.end, s.front_tiles); ++t) f.rows(g, g.front, head, t * kTile, g.front.rows, g.front.rows);
    for (int32_t t = max(s.begin, s.front_tiles); t < min(s.end, stored_end); ++t) f.stored(g, head, t - s.front_tiles);
    for (int32_t t = max(s.begin, stored_end); t < s.end; ++t) f.rows(g, g.recent, head, (t - stored_end) * kTile, recent, seen);

    float sum = f.sum;
    sum += lane_xor<16>(sum);
    sum += lane_xor<32>(sum);
    if constexpr (Form::RAISED != 0.0f) {
        sum *= 0x1p-15f;
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) f.o[n] *= 0x1p-15f;
    }
    if (!there) return;
    // the lane holds channels run(v) + VU * (4 * quarter + i) + 0 .. VU - 1 of its query row
    const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
    const int64_t at = (int64_t)q_head * g.t_q + token;
#pragma unroll
    for (int v = 0; v < Form::VN; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = v * 16 * Form::VU + (4 * quarter + i) * Form::VU;
            if (c >= g.channels) continue;
            float x[Form::VU];
#pragma unroll
            for (int n = 0; n < Form::VU; ++n) x[n] = f.o[v * Form::VU + n][i];
            if (g.splits > 1) {
                float* p = g.part_out + (at * g.splits + cut) * g.channels + c;
#pragma unroll
                for (int n = 0; n < Form::VU; n += 4) *reinterpret_cast<f32x4*>(p + n) = f32x4{x[n], x[n + 1], x[n + 2], x[n + 3]};
            } else {
                typedef typename Element<T>::type E;
                typedef E Vec __attribute__((ext_vector_type(Form::VU)));
                Vec y;
#pragma unroll
                for (int n = 0; n < Form::VU; ++n) y[n] = (E)(x[n] * by);
                *reinterpret_cast<Vec*>(g.out + q_head * g.out_head + token * g.out_row + (int64_t)c * sizeof(E)) = y;
            }
        }
    if (quarter == 0) {
        if (g.splits > 1) g.part_stat[at * g.splits + cut] = f32pair{f.top, sum};
        else if (g.lse) g.lse[at] = sum > 0.0f ? (f.top * g.score_unit + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
    }
}

// ---- joining the parts ---------------------------------------------------------------------------------------------------------
// The rows of the parts, weighted by 2^(M_s - M), and the sum of their sums.  A lane takes four channels and some of the parts, with
// the running maximum again, so that no load waits for another; four parts are in flight.
struct Joined {
    float top = -__builtin_inff(), total = 0.0f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float unit, float their_top, float their_total, const f32x4& their_sum) {
        const float next = fmaxf(top, their_top), from = next == -__builtin_inff() ? 0.0f : next;
        const float mine = exp2_of((top - from) * unit), theirs = exp2_of((their_top - from) * unit);
        top = next;
        total = total * mine + their_total * theirs;
        sum = sum * mine + their_sum * theirs;
    }
};
template <typename T>
__device__ __forceinline__ void put_joined(const AttendArgs& g, int64_t at, int c, const Joined& j) {
    const int32_t q_head = (int32_t)(at / g.t_q), token = (int32_t)(at - (int64_t)q_head * g.t_q);
    const float by = j.total > 0.0f ? 1.0f / j.total : 0.0f;
    typedef typename Element<T>::type E;
    typedef E Vec __attribute__((ext_vector_type(4)));
    Vec y;
#pragma unroll
    for (int n = 0; n < 4; ++n) y[n] = (E)(j.sum[n] * by);
    *reinterpret_cast<Vec*>(g.out + q_head * g.out_head + token * g.out_row + (int64_t)c * sizeof(E)) = y;
    if (c == 0 && g.lse) g.lse[at] = j.total > 0.0f ? (j.top * g.score_unit + __builtin_amdgcn_logf(j.total)) * kLn2 : -__builtin_inff();
}
constexpr int kJoinAhead = 4;
__device__ __forceinline__ Joined join_parts(const AttendArgs& g, int64_t at, int c, int first, int step) {
    const f32pair* stat = g.part_stat + at * g.splits;
    const float* part = g.part_out + at * g.splits * g.channels + c;
    Joined j;
    for (int s0 = first; s0 < g.splits; s0 += step * kJoinAhead) {
        f32pair st[kJoinAhead];
        f32x4 x[kJoinAhead];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
            const int s = min(s0 + u * step, g.splits - 1);  // behind the last: read again, and not added
            st[u] = stat[s];
            x[u] = *reinterpret_cast<const f32x4*>(part + (int64_t)s * g.channels);
        }
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            if (s0 + u * step < g.splits) j.add(g.score_unit, st[u].x, st[u].y, x[u]);
    }
    return j;
}
// What the lane N on, or back, has found.
template <int N>
__device__ __forceinline__ void join_across(const AttendArgs& g, Joined& j) {
    const float top = lane_xor<N>(j.top), total = lane_xor<N>(j.total);
    f32x4 sum;
#pragma unroll
    for (int n = 0; n < 4; ++n) sum[n] = lane_xor<N>(j.sum[n]);
    j.add(g.score_unit, top, total, sum);
}
// Few parts: a lane takes them all.
template <typename T>
__global__ __launch_bounds__(kBlock) void attend_join_few_kernel(AttendArgs g, uint32_t lanes, uint32_t inv_lanes, uint32_t rows) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x, row = div_by(i, lanes, inv_lanes);
    if (row >= rows) return;
    const int c = 4 * (int)(i - row * lanes);
    put_joined<T>(g, row, c, join_parts(g, row, c, 0, 1));
}
// Many: a workgroup takes 32 channels of a row, eight lanes to a part, and joins what its lanes found.
template <typename T>
__global__ __launch_bounds__(kBlock) void attend_join_many_kernel(AttendArgs g) {
    constexpr int kLanes = 8, kSets = kBlock / kLanes;
    const int lane = (int)threadIdx.x % kLanes, set = (int)threadIdx.x / kLanes;
    const int c = 4 * ((int)blockIdx.y * kLanes + lane);
    const bool there = c < g.channels;
    Joined j;
    if (there) j = join_parts(g, blockIdx.x, c, set, kSets);
    join_across<8>(g, j);
    join_across<16>(g, j);
    join_across<32>(g, j);
    __shared__ float tops[kBlock / 64][kLanes], totals[kBlock / 64][kLanes];
    __shared__ f32x4 sums[kBlock / 64][kLanes];
    const int wave = (int)threadIdx.x / 64;
    if ((int)threadIdx.x % 64 < kLanes) {
        tops[wave][lane] = j.top;
        totals[wave][lane] = j.total;
        sums[wave][lane] = j.sum;
    }
    __syncthreads();
    if (threadIdx.x >= kLanes || !there) return;
    for (int w = 1; w < kBlock / 64; ++w) j.add(g.score_unit, tops[w][lane], totals[w][lane], sums[w][lane]);
    put_joined<T>(g, blockIdx.x, c, j);
}
// A lane takes all parts where they are few, or where the rows alone fill the chip: eight lanes to a part then only read the
// same bytes by more workgroups. Whole call at 128 channels, a lane takes all / workgroups: 28 rows of 4, 6, 8, 12, 24 parts 7.9,
// 8.8, 9.4, 9.6, 12.2 / 8.2, 8.2, 9.0, 8.6, 8.7 us; 448 rows of 25 30.3 / 27.8; 896 of 48 76.3 / 71.3; 1680 of 13 28.6 / 32.9;
// 1792 of 27 111.1 / 113.3; 5040 of 9 43.3 / 61.3; 28000 of 5 175 / 283.
constexpr int kFewParts = 4;
constexpr uint32_t kLanesThatFill = 48 * 1024;
template <typename T>
void start_join(const AttendArgs& g, hipStream_t s) {
    const uint32_t rows = (uint32_t)(g.kv_heads * g.repeat * g.t_q), lanes = (uint32_t)(g.channels / 4);
    if (g.splits <= kFewParts || rows * lanes >= kLanesThatFill) {
        // calls that are cut into parts have at most 2047 workgroups of 64 rows: rows * lanes stays below 2^23
        launch(attend_join_few_kernel<T>, dim3((rows * lanes + kBlock - 1) / kBlock), dim3(kBlock), 0, s, g, lanes, reciprocal_u32(lanes), rows);
    } else {
        launch(attend_join_many_kernel<T>, dim3(rows, (lanes + 7) / 8), dim3(kBlock), 0, s, g);
    }
}

template <typename T>
void start_general(const AttendArgs& g, hipStream_t s) {
    const uint64_t items = (uint64_t)g.row_blocks * (uint64_t)g.splits * (uint64_t)g.kv_heads;
    const dim3 grid((uint32_t)((items + kBlock / 64 - 1) / (kBlock / 64))), block(kBlock);
    if (g.channels <= 64) launch(g.token_axis ? attend_kernel<T, 64, true> : attend_kernel<T, 64, false>, grid, block, 0, s, g);
    else if (g.channels <= 128) launch(g.token_axis ? attend_kernel<T, 128, true> : attend_kernel<T, 128, false>, grid, block, 0, s, g);
    else launch(g.token_axis ? attend_kernel<T, 256, true> : attend_kernel<T, 256, false>, grid, block, 0, s, g);
}

hipError_t launch_attend(const AttendArgs& g, const AttendForm& form, int dtype, hipStream_t s) {
    if (form.shared) {
        (dtype == TOM_BF16 ? start_attend_shared_bf16 : start_attend_shared_f16)(g, s);
    } else if (form.folded) {
        if (dtype == TOM_BF16) (g.bits == 4 ? start_attend_bf16_4bit : start_attend_bf16_2bit)(g, form, s);
        else (g.bits == 4 ? start_attend_f16_4bit : start_attend_f16_2bit)(g, form, s);
    } else if (dtype == TOM_F32) {
        start_general<In_f32>(g, s);
    } else if (dtype == TOM_BF16) {
        start_general<In_bf16>(g, s);
    } else {
        start_general<In_f16>(g, s);
    }
    if (g.splits > 1) {
        if (dtype == TOM_F32) start_join<In_f32>(g, s);
        else if (dtype == TOM_BF16) start_join<In_bf16>(g, s);
        else start_join<In_f16>(g, s);
    }
    return hipGetLastError();
}

}  // namespace oqm
