// Attention of new tokens over rows in front, stored groups as they are stored, and recent rows, in one softmax.
//
//   w_j = scale <q, k_j> (or softcap tanh of it / softcap)      out = sum_j exp(w_j - M) v_j / sum_j exp(w_j - M)
//
// One pass over the keys and values with the running maximum and sum of each query row.  The keys' product is taken transposed,
// S^T = K Q^T on the matrix cores: a lane then holds, for one query row, the scores of the very tokens whose values it feeds as
// the other operand of O^T = V^T P^T, so that the probabilities never leave their lane.
#include "oqm_attend_device.h"

namespace oqm {

__device__ __forceinline__ f32x2 load_pair(const char* meta, int64_t i, bool bf16) {
    if (bf16) return widen_pair(reinterpret_cast<const uint32_t*>(meta)[i]);
    return reinterpret_cast<const f32x2*>(meta)[i];
}

// N consecutive channels from c of token `tok` of a stored head tile.
template <int N>
__device__ __forceinline__ void load_stored(const AttendArgs& g, const char* codes, const char* meta, uint32_t tok, int c, float* x) {
    const int64_t first = ((int64_t)tok * g.channels + c) * g.bits / 8;
    uint32_t w;
    if (g.bits == 4) w = N == 8 ? *reinterpret_cast<const uint32_t*>(codes + first) : *reinterpret_cast<const uint16_t*>(codes + first);
    else w = N == 8 ? *reinterpret_cast<const uint16_t*>(codes + first) : *reinterpret_cast<const uint8_t*>(codes + first);
    const uint32_t mask = g.bits == 4 ? 15u : 3u;
    if (g.token_axis) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const f32x2 p = load_pair(meta, c + i, g.meta_bf16 != 0);
            x[i] = __builtin_fmaf((float)((w >> (g.bits * i)) & mask), p[0], p[1]);
        }
    } else {
        const f32x2 p = load_pair(meta, ((int64_t)tok * g.channels + c) >> g.qgroup_log2, g.meta_bf16 != 0);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_fmaf((float)((w >> (g.bits * i)) & mask), p[0], p[1]);
    }
}

// Where a token of the groups' rows stands: its slot (-1: a hole, or no token) and its row in the group.
__device__ __forceinline__ int32_t locate(const AttendArgs& g, int32_t token, int32_t tokens, uint32_t& tok) {
    tok = 0;
    if (token >= tokens) return -1;
    const uint32_t rank = div_by((uint32_t)token, (uint32_t)g.group_tokens, g.inv_group_tokens);
    tok = (uint32_t)token - rank * (uint32_t)g.group_tokens;
    const int32_t slot = g.idx ? g.idx[rank] : (int32_t)rank;
    return slot >= 0 && slot < g.n_groups ? slot : -1;
}

// ---- general form ------------------------------------------------------------------------------------------------------------
// A wave takes 16 query rows of a KV head and a run of 32-token tiles, on its own: every element is reconstructed (or widened) to
// float32 and enters the products in two 16-bit parts where one does not hold it.  DP: channels, padded with zeros.
//   K operand  lane (token l % 16 of a half, quarter l / 16): DP / 4 consecutive channels
//   V operand  lane (l % 16, l / 16): of the 8 tokens whose scores it holds, VN runs of VU channels
template <typename T, int DP>
struct General {
    static constexpr int VU = DP / 16 < 8 ? DP / 16 : 8, VN = DP / 16 / VU, STEPS = DP / 32;
    Operand<T> q[STEPS];
    f32x4 o[DP / 16];
    float top, sum;

    // STORED: a tile of the groups' rows; else of `r`.  `seen`: of the rows from the first, how many the lane's query row sees.
    template <bool STORED>
    __device__ __forceinline__ void tile(const AttendArgs& g, const AttendRows* r, int head, int32_t t0, int32_t tokens, int32_t seen) {
        const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
        const char *kc = nullptr, *km = nullptr, *vc = nullptr, *vm = nullptr;
        if constexpr (STORED) {
            kc = g.codes[0] + head * g.code_head;
            vc = g.codes[1] + head * g.code_head;
            km = g.meta[0] + head * g.meta_head;
            vm = g.meta[1] + head * g.meta_head;
        } else {
            kc = r->k + head * r->k_head;
            vc = r->v + head * r->v_head;
        }
        float w[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int32_t token = t0 + 16 * half + a;
            uint32_t tok = 0;
            int32_t slot = token < tokens ? token : -1;
            if constexpr (STORED) slot = locate(g, token, tokens, tok);
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int c = quarter * (DP / 4) + 8 * u;
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 0.0f;
                if (slot >= 0 && c < g.channels) {
                    if constexpr (STORED) load_stored<8>(g, kc + slot * g.code_slot, km + slot * g.meta_slot, tok, c, x);
                    else load_row<T, 8>(kc + slot * r->k_row + (int64_t)c * elem_bytes<T>::value, x);
                }
                Operand<T> hi, lo;
                split(x, hi, lo);
                s = product(hi, q[u], s);
                if constexpr (STORED && !__is_same(T, In_f32)) s = product(lo, q[u], s);
            }
            const uint32_t there = (uint32_t)(__ballot(slot >= 0) & 0xffff);  // of the half's 16 tokens
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * quarter + i;
                const float y = s[i] * g.scale_log2;
                const float z = g.cap_log2 != 0.0f ? capped_exactly(y, g.cap_log2) : y;
                w[4 * half + i] = (there >> j & 1u) && t0 + 16 * half + j < seen ? z : -__builtin_inff();
            }
        }
        float high = w[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) high = fmaxf(high, w[i]);
        high = fmaxf(high, __shfl_xor(high, 16, 64));
        high = fmaxf(high, __shfl_xor(high, 32, 64));
        if (__any(high > top)) {
            const float next = fmaxf(top, high);
            const float by = next == -__builtin_inff() ? 1.0f : exp2_of(top - next);
            top = next;
            sum *= by;
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) o[n] *= by;
        }
        const float from = top == -__builtin_inff() ? 0.0f : top;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = exp2_of(w[i] - from);
            sum += p[i];
        }
        Operand<T> ph, pl;
        split(p, ph, pl);
#pragma unroll
        for (int v = 0; v < VN; ++v) {
            const int c = v * 16 * VU + a * VU;
            float x[8][VU];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
#pragma unroll
                for (int i = 0; i < VU; ++i) x[j][i] = 0.0f;
                const int32_t token = t0 + 16 * (j / 4) + 4 * quarter + j % 4;
                uint32_t tok = 0;
                int32_t slot = token < tokens ? token : -1;
                if constexpr (STORED) slot = locate(g, token, tokens, tok);
                if (slot >= 0 && c < g.channels) {
                    if constexpr (STORED) load_stored<VU>(g, vc + slot * g.code_slot, vm + slot * g.meta_slot, tok, c, x[j]);
                    else load_row<T, VU>(vc + slot * r->v_row + (int64_t)c * elem_bytes<T>::value, x[j]);
                }
            }
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j][i];
                Operand<T> hi, lo;
                split(y, hi, lo);
                f32x4& acc = o[v * VU + i];
                acc = product(hi, ph, acc);
                if constexpr (!__is_same(T, In_f32)) {
                    acc = product(hi, pl, acc);
                    if constexpr (STORED) acc = product(lo, ph, acc);
                }
            }
        }
    }
};

template <typename T, int DP>
__global__ __launch_bounds__(kBlock) void attend_kernel(AttendArgs g) {
    typedef General<T, DP> Form;
    const uint32_t item = blockIdx.x * (kBlock / 64) + threadIdx.x / 64;
    const uint32_t block = item % (uint32_t)g.row_blocks, rest = item / (uint32_t)g.row_blocks;
    const uint32_t cut = rest % (uint32_t)g.splits;
    const int head = (int)(rest / (uint32_t)g.splits);
    if (head >= g.kv_heads) return;
    const int lane = (int)__lane_id(), a = lane & 15, quarter = lane >> 4;
    // query rows of a KV head: token-major, so that a block of them ends at about one token
    const int32_t rows = g.t_q * g.repeat;
    const int32_t row = (int32_t)block * 16 + a;
    const bool there = row < rows;
    const int32_t token = there ? (int32_t)div_by((uint32_t)row, (uint32_t)g.repeat, g.inv_repeat) : 0;
    const int32_t q_head = head * g.repeat + (there ? row - token * g.repeat : 0);

    Form f;
    f.top = -__builtin_inff();
    f.sum = 0.0f;
#pragma unroll
    for (int n = 0; n < DP / 16; ++n) f.o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < Form::STEPS; ++u) {
        const int c = quarter * (DP / 4) + 8 * u;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        if (there && c < g.channels) load_row<T, 8>(g.q + q_head * g.q_head + token * g.q_row + (int64_t)c * elem_bytes<T>::value, x);
        Operand<T> unused;
        split(x, f.q[u], unused);
    }

    const int32_t stored = g.k_eff * g.group_tokens;
    const int32_t last_token = min((int32_t)block * 16 + 15, rows - 1) / g.repeat;
    int32_t recent = g.recent.rows;  // as far as any row of the block sees
    if (g.causal) recent = max(0, min(recent, last_token + 1 + g.recent.rows - g.t_q));
    const int32_t seen = !there ? 0 : g.causal ? token + 1 + g.recent.rows - g.t_q : g.recent.rows;
    const int32_t front_tiles = (g.front.rows + kTile - 1) / kTile, stored_tiles = (stored + kTile - 1) / kTile;
    const int32_t tiles = front_tiles + stored_tiles + (recent + kTile - 1) / kTile;
    const int32_t begin = (int32_t)((int64_t)tiles * cut / g.splits), end = (int32_t)((int64_t)tiles * (cut + 1) / g.splits);
    for (int32_t t = begin; t < min(end, front_tiles); ++t)
        f.template tile<false>(g, &g.front, head, t * kTile, g.front.rows, there ? g.front.rows : 0);
    for (int32_t t = max(begin, front_tiles); t < min(end, front_tiles + stored_tiles); ++t)
        f.template tile<true>(g, nullptr, head, (t - front_tiles) * kTile, stored, there ? stored : 0);
    for (int32_t t = max(begin, front_tiles + stored_tiles); t < end; ++t)
        f.template tile<false>(g, &g.recent, head, (t - front_tiles - stored_tiles) * kTile, recent, seen);

    float sum = f.sum;
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
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
        else if (g.lse) g.lse[at] = sum > 0.0f ? (f.top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
    }
}

// ---- joining the parts ---------------------------------------------------------------------------------------------------------
// The rows of the parts, weighted by 2^(M_s - M), and the sum of their sums.  A lane takes four channels and some of the parts, with
// the running maximum again, so that no load waits for another; four parts are in flight.
struct Joined {
    float top = -__builtin_inff(), total = 0.0f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float their_top, float their_total, const f32x4& their_sum) {
        const float next = fmaxf(top, their_top), from = next == -__builtin_inff() ? 0.0f : next;
        const float mine = exp2_of(top - from), theirs = exp2_of(their_top - from);
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
    if (c == 0 && g.lse) g.lse[at] = j.total > 0.0f ? (j.top + __builtin_amdgcn_logf(j.total)) * kLn2 : -__builtin_inff();
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
            if (s0 + u * step < g.splits) j.add(st[u].x, st[u].y, x[u]);
    }
    return j;
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
#pragma unroll
    for (int m = kLanes; m < 64; m *= 2) {
        const float top = __shfl_xor(j.top, m, 64), total = __shfl_xor(j.total, m, 64);
        f32x4 sum;
#pragma unroll
        for (int n = 0; n < 4; ++n) sum[n] = __shfl_xor(j.sum[n], m, 64);
        j.add(top, total, sum);
    }
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
    for (int w = 1; w < kBlock / 64; ++w) j.add(tops[w][lane], totals[w][lane], sums[w][lane]);
    put_joined<T>(g, blockIdx.x, c, j);
}
// Up to this many parts a lane takes them all.
constexpr int kFewParts = 8;
template <typename T>
void start_join(const AttendArgs& g, hipStream_t s) {
    const uint32_t rows = (uint32_t)(g.kv_heads * g.repeat * g.t_q), lanes = (uint32_t)(g.channels / 4);
    if (g.splits <= kFewParts) {
        // parts are cut from calls of 2048 waves of 16 rows or less: rows * lanes stays far inside 32 bits
        launch(attend_join_few_kernel<T>, dim3((rows * lanes + kBlock - 1) / kBlock), dim3(kBlock), 0, s, g, lanes, reciprocal_u32(lanes), rows);
    } else {
        launch(attend_join_many_kernel<T>, dim3(rows, (lanes + 7) / 8), dim3(kBlock), 0, s, g);
    }
}

template <typename T>
void start_general(const AttendArgs& g, hipStream_t s) {
    const uint64_t items = (uint64_t)g.row_blocks * (uint64_t)g.splits * (uint64_t)g.kv_heads;
    const dim3 grid((uint32_t)((items + kBlock / 64 - 1) / (kBlock / 64))), block(kBlock);
    if (g.channels <= 64) launch(attend_kernel<T, 64>, grid, block, 0, s, g);
    else if (g.channels <= 128) launch(attend_kernel<T, 128>, grid, block, 0, s, g);
    else launch(attend_kernel<T, 256>, grid, block, 0, s, g);
}

hipError_t launch_attend(const AttendArgs& g, const AttendForm& form, int dtype, hipStream_t s) {
    if (form.folded) {
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
