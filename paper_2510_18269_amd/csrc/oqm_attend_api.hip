// Host side of tom_oqm_attend: validation, and how the call is cut over the chip.  Nothing here allocates device memory or
// synchronises with the GPU.
#include <cmath>

#include "oqm_attend.h"

namespace oqm {

static int bytes_of(int32_t dtype) { return dtype == TOM_F32 ? 4 : 2; }

constexpr int32_t kMaxNewTokens = 1 << 20;
constexpr int64_t kMaxRows = 0x7fffffff - 4096;  // a tile's last token stays inside 32 bits

static size_t part_bytes(const tom_oqm_config_t& c, int32_t t_q, int32_t splits) {
    if (splits <= 1) return 0;
    return (size_t)c.n_q_heads * (size_t)t_q * (size_t)splits * ((size_t)c.head_dim * sizeof(float) + sizeof(f32pair));
}

// A strided view as the call wants it; sizes of one make their stride meaningless.
static tom_status_t check_view(const tom_oqm_view_t* v, const char* name, int32_t heads, int32_t rows, const tom_oqm_config_t& c,
                               int64_t& head_bytes, int64_t& row_bytes) {
    constexpr int64_t kMaxStride = int64_t{1} << 40;  // elements; far beyond any device tensor
    if (v->dtype != c.out_dtype) return fail(TOM_ERR_INVALID_ARG, "the dtype of %s is not the memory's out_dtype", name);
    if (v->heads != heads || v->channels != c.head_dim || v->rows != rows)
        return fail(TOM_ERR_INVALID_ARG, "%s is [%d][%d][%d], wanted [%d][%d][%d]", name, v->heads, v->rows, v->channels, heads, rows, c.head_dim);
    const int e = bytes_of(v->dtype);
    if (v->head_stride < 0 || v->row_stride < 0 || v->head_stride > kMaxStride || v->row_stride > kMaxStride)
        return fail(TOM_ERR_INVALID_ARG, "strides of %s must be in [0, 2^40] elements", name);
    head_bytes = heads > 1 ? v->head_stride * e : 0;
    row_bytes = rows > 1 ? v->row_stride * e : 0;
    if (!v->data) return fail(TOM_ERR_INVALID_ARG, "%s has no data", name);
    if ((reinterpret_cast<uintptr_t>(v->data) | (uintptr_t)head_bytes | (uintptr_t)row_bytes) & 15u)
        return fail(TOM_ERR_INVALID_ARG, "%s and its strides must be multiples of 16 bytes", name);
    return TOM_OK;
}

static tom_status_t check_rows(const tom_oqm_view_t* k, const tom_oqm_view_t* v, const char* k_name, const char* v_name,
                               const tom_oqm_config_t& c, AttendRows& r) {
    const int32_t rows = k ? k->rows : 0;
    if ((v ? v->rows : 0) != rows) return fail(TOM_ERR_INVALID_ARG, "%s and %s must have the same rows", k_name, v_name);
    if (rows < 0) return fail(TOM_ERR_INVALID_ARG, "%s has a negative size", k_name);
    if (rows == 0) return TOM_OK;
    if (tom_status_t st = check_view(k, k_name, c.n_kv_heads, rows, c, r.k_head, r.k_row)) return st;
    if (tom_status_t st = check_view(v, v_name, c.n_kv_heads, rows, c, r.v_head, r.v_row)) return st;
    r.k = static_cast<const char*>(k->data);
    r.v = static_cast<const char*>(v->data);
    r.rows = rows;
    return TOM_OK;
}

}  // namespace oqm

using namespace oqm;

extern "C" {

size_t tom_oqm_attend_workspace_bytes(const tom_oqm_t* h, int32_t t_q, int64_t rows) {
    if (!h || t_q < 1 || t_q > kMaxNewTokens || rows < 0 || rows > kMaxRows || h->cfg.head_dim > 256) return 0;
    return part_bytes(h->cfg, t_q, attend_cuts(h->cfg, t_q, rows));
}

tom_status_t tom_oqm_attend(const tom_oqm_t* h, int32_t layer, const tom_oqm_view_t* q, const tom_oqm_view_t* out, const int32_t* idx,
                            int32_t k_eff, const tom_oqm_view_t* front_k, const tom_oqm_view_t* front_v, const tom_oqm_view_t* recent_k,
                            const tom_oqm_view_t* recent_v, int32_t causal, float scale, float softcap, float* lse, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
    if (!h) return fail(TOM_ERR_INVALID_ARG, "handle is NULL");
    const tom_oqm_config_t& c = h->cfg;
    if (layer < 0 || layer >= c.n_layers) return fail(TOM_ERR_INVALID_ARG, "layer %d is outside [0, %d)", layer, c.n_layers);
    if (!q || !out) return fail(TOM_ERR_INVALID_ARG, "q and out must be non-NULL");
    const int32_t t_q = q->rows;
    if (t_q < 0) return fail(TOM_ERR_INVALID_ARG, "q has a negative size");
    if (k_eff < 0) return fail(TOM_ERR_INVALID_ARG, "k_eff < 0");
    if (k_eff > 0 && !h->bound) return fail(TOM_ERR_NOT_BOUND, "tom_oqm_bind has not been called");
    if (!idx && k_eff > h->n_groups)
        return fail(TOM_ERR_INVALID_ARG, "k_eff = %d without an idx exceeds the %d stored groups", k_eff, h->n_groups);
    if ((reinterpret_cast<uintptr_t>(idx) & 3u) != 0) return fail(TOM_ERR_INVALID_ARG, "idx must be 4-byte aligned");
    if (!is_number(scale)) return fail(TOM_ERR_INVALID_ARG, "scale must be a number");
    if (!is_number(softcap) || softcap < 0.0f) return fail(TOM_ERR_INVALID_ARG, "softcap must be a number >= 0");
    if (c.head_dim > 256) return fail(TOM_ERR_UNSUPPORTED, "head_dim %d: the attention covers 256 and less", c.head_dim);
    if (t_q > kMaxNewTokens) return fail(TOM_ERR_UNSUPPORTED, "%d new tokens: at most %d per call", t_q, kMaxNewTokens);
    AttendArgs a{};
    if (t_q == 0) return TOM_OK;
    if (tom_status_t st = check_view(q, "q", c.n_q_heads, t_q, c, a.q_head, a.q_row)) return st;
    if (tom_status_t st = check_view(out, "out", c.n_q_heads, t_q, c, a.out_head, a.out_row)) return st;
    if (!elements_apart(*out)) return fail(TOM_ERR_INVALID_ARG, "heads or rows of out overlap");
    if (tom_status_t st = check_rows(front_k, front_v, "front_k", "front_v", c, a.front)) return st;
    if (tom_status_t st = check_rows(recent_k, recent_v, "recent_k", "recent_v", c, a.recent)) return st;
    const int64_t rows = (int64_t)a.front.rows + (int64_t)k_eff * c.group_tokens + a.recent.rows;
    if (rows > kMaxRows) return fail(TOM_ERR_UNSUPPORTED, "%lld rows: at most %lld per call", (long long)rows, (long long)kMaxRows);
    const AttendForm form = attend_form(c, t_q);
    a.splits = attend_cuts(c, t_q, rows);
    const int64_t blocks = ((int64_t)(c.n_q_heads / c.n_kv_heads) * t_q + form.rows - 1) / form.rows;
    // (so that the query rows of a KV head, rounded up to whole blocks, stay inside 32 bits too)
    if (attend_lanes(form, (uint64_t)blocks * (uint64_t)a.splits * (uint64_t)c.n_kv_heads) > kMaxLanes)
        return fail(TOM_ERR_UNSUPPORTED, "%d heads of %d queries need more lanes than the 2^32 - 1 of a launch", c.n_q_heads, t_q);
    const size_t need = part_bytes(c, t_q, a.splits);
    if (need > 0) {
        if (!workspace || workspace_bytes < need)
            return fail(TOM_ERR_INVALID_ARG, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
        if ((reinterpret_cast<uintptr_t>(workspace) & 15u) != 0) return fail(TOM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
        a.part_out = static_cast<float*>(workspace);
        a.part_stat = reinterpret_cast<f32pair*>(a.part_out + (size_t)c.n_q_heads * t_q * a.splits * c.head_dim);
    }
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return fail(TOM_ERR_INVALID_ARG, "lse must be 4-byte aligned");

    const Layout lay = layout_of(c);
    const int64_t pair_bytes = c.meta_dtype == TOM_BF16 ? 4 : 8;
    a.code_head = lay.tile_code_bytes;
    a.meta_head = lay.tile_meta * pair_bytes;
    a.code_slot = a.code_head * c.n_kv_heads;
    a.meta_slot = a.meta_head * c.n_kv_heads;
    for (int kv = 0; kv < 2 && k_eff > 0; ++kv) {
        const int64_t plane = ((int64_t)layer * 2 + kv) * c.capacity_groups;
        a.codes[kv] = reinterpret_cast<const char*>(h->codes) + plane * a.code_slot;
        a.meta[kv] = static_cast<const char*>(h->meta) + plane * a.meta_slot;
    }
    a.idx = idx;
    a.q = static_cast<const char*>(q->data);
    a.out = static_cast<char*>(out->data);
    a.lse = lse;
    a.k_eff = k_eff;
    a.n_groups = h->n_groups;
    a.group_tokens = c.group_tokens;
    a.inv_group_tokens = reciprocal_u32((uint32_t)c.group_tokens);
    a.channels = c.head_dim;
    if (c.qaxis == TOM_QAXIS_HEAD_DIM)
        while ((1 << a.qgroup_log2) < c.qgroup) ++a.qgroup_log2;
    a.t_q = t_q;
    a.repeat = c.n_q_heads / c.n_kv_heads;
    a.inv_repeat = reciprocal_u32((uint32_t)a.repeat);
    a.kv_heads = c.n_kv_heads;
    a.causal = causal != 0;
    a.token_axis = c.qaxis == TOM_QAXIS_TOKENS;
    a.bits = c.bits;
    a.meta_bf16 = c.meta_dtype == TOM_BF16;
    // Under a cap below 2^-30 all scores are zero to float32's last place beside the one of exp(0); one above 2^40 changes none of up to 2^28.
    if (softcap > 0.0f && softcap < 0x1p-30f) scale = softcap = 0.0f;
    if (softcap > 0x1p40f) softcap = 0.0f;
    // what the folded form multiplies scales by stays finite
    if (std::fabs(softcap > 0.0f ? scale / softcap : scale) >= 0x1p50f)
        return fail(TOM_ERR_INVALID_ARG, "scale, or scale / softcap, must be below 2^50");
    constexpr float kLog2e = 1.4426950408889634f;
    a.scale_log2 = softcap > 0.0f ? 2.0f * kLog2e * scale / softcap : scale * kLog2e;
    a.score_unit = 1.0f;
    if (!form.folded && !form.shared && softcap == 0.0f && scale != 0.0f) {
        a.score_unit = std::fabs(a.scale_log2);
        a.scale_log2 = scale > 0.0f ? 1.0f : -1.0f;
    }
    a.cap_log2 = softcap * kLog2e;
    a.row_blocks = (int32_t)blocks;
    a.inv_row_blocks = reciprocal_u32((uint32_t)a.row_blocks);
    a.inv_splits = reciprocal_u32((uint32_t)a.splits);
    (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
    const hipError_t err = launch_attend(a, form, c.out_dtype, static_cast<hipStream_t>(hip_stream));
    if (err != hipSuccess) return fail(TOM_ERR_HIP, "attend launch: %s", hipGetErrorString(err));
    return TOM_OK;
}

}  // extern "C"
