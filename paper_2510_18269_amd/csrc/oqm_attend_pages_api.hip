// Host side of tom_oqm_attend_pages: validation, and how the call is cut over the chip.  Nothing here allocates device memory or
// synchronises with the GPU.
#include <cmath>

#include "oqm_attend_pages.h"

namespace oqm {

constexpr int32_t kMaxNewTokens = 1 << 20;

// Bytes of the workspace's three arrays, each a multiple of 16.
struct PagesWorkspace {
    size_t out, stat, units;
    size_t all() const { return out + stat + units; }
};
static PagesWorkspace workspace_of(const tom_oqm_pages_t& g, const PagesForm& f, const PagesCuts& c) {
    if (c.extra == 0) return {0, 0, 0};
    const size_t rows = (size_t)c.items * (size_t)g.heads * (size_t)f.block_rows;
    return {rows * (size_t)g.channels * sizeof(float), (rows * sizeof(f32pair) + 15) / 16 * 16, ((size_t)c.units * 8 + 15) / 16 * 16 + 16};
}

// A strided view as the call wants it; sizes of one make their stride meaningless.  Strides in units of `unit` bytes.
static tom_status_t check_view(const tom_oqm_view_t* v, const char* name, int32_t heads, int32_t rows, int32_t channels, int32_t dtype, int64_t align, int64_t unit,
                               int64_t& head_step, int64_t& row_step) {
    constexpr int64_t kMaxStride = int64_t{1} << 40;  // elements; far beyond any device tensor
    if (v->dtype != dtype) return fail(TOM_ERR_INVALID_ARG, "%s has another dtype than the call wants", name);
    if (v->heads != heads || v->channels != channels || v->rows != rows)
        return fail(TOM_ERR_INVALID_ARG, "%s is [%d][%d][%d], wanted [%d][%d][%d]", name, v->heads, v->rows, v->channels, heads, rows, channels);
    if (v->head_stride < 0 || v->row_stride < 0 || v->head_stride > kMaxStride || v->row_stride > kMaxStride)
        return fail(TOM_ERR_INVALID_ARG, "strides of %s must be in [0, 2^40] elements", name);
    const int64_t e = bytes_of_dtype(dtype);
    const int64_t head = heads > 1 ? v->head_stride * e : 0, row = rows > 1 ? v->row_stride * e : 0;
    if (!v->data) return fail(TOM_ERR_INVALID_ARG, "%s has no data", name);
    if ((reinterpret_cast<uintptr_t>(v->data) | (uintptr_t)head | (uintptr_t)row) & (uintptr_t)(align - 1))
        return fail(TOM_ERR_INVALID_ARG, "%s and its strides must be multiples of %d bytes", name, (int)align);
    head_step = head / unit;
    row_step = row / unit;
    return TOM_OK;
}

hipError_t launch_attend_pages(const PagesArgs& g, const PagesForm& form, int dtype, hipStream_t s) {
    if (dtype == TOM_F32) start_attend_pages_f32(g, form, s);
    else if (dtype == TOM_BF16) start_attend_pages_bf16(g, form, s);
    else start_attend_pages_f16(g, form, s);
    return hipGetLastError();
}

}  // namespace oqm

using namespace oqm;

extern "C" {

size_t tom_oqm_attend_pages_workspace_bytes(const tom_oqm_pages_t* pages, int32_t tokens, int32_t n_q_heads) {
    PagePlaces p;
    if (check_pages(pages, p) != TOM_OK || tokens < 1 || tokens > kMaxNewTokens || pages->sequences < 1 || n_q_heads < 1 || n_q_heads % pages->heads ||
        (!pages->starts && tokens != pages->sequences) || (int64_t)n_q_heads * tokens >= 1 << 30)
        return 0;
    const PagesForm f = pages_form(*pages, tokens, n_q_heads);
    return workspace_of(*pages, f, pages_cuts(*pages, tokens, n_q_heads, f)).all();
}

tom_status_t tom_oqm_attend_pages(const tom_oqm_pages_t* pages, int32_t layer, const tom_oqm_view_t* q, const tom_oqm_view_t* out, const int64_t* mask, int32_t words,
                                  int32_t causal, float scale, float softcap, const tom_oqm_view_t* prior_out, const tom_oqm_view_t* prior_lse,
                                  const tom_oqm_view_t* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    PagesArgs a{};
    if (tom_status_t st = check_pages(pages, a.p)) return st;
    if (layer < 0 || layer >= pages->n_layers) return fail(TOM_ERR_INVALID_ARG, "layer %d is outside [0, %d)", layer, pages->n_layers);
    if (!q || !out) return fail(TOM_ERR_INVALID_ARG, "q and out must be non-NULL");
    const int32_t tokens = q->rows, n_q_heads = q->heads, channels = pages->channels;
    if (tokens < 0) return fail(TOM_ERR_INVALID_ARG, "q has a negative size");
    if (n_q_heads < 1 || n_q_heads % pages->heads) return fail(TOM_ERR_INVALID_ARG, "%d query heads are no multiple of the pages' %d", n_q_heads, pages->heads);
    if (!prior_out != !prior_lse) return fail(TOM_ERR_INVALID_ARG, "prior_out and prior_lse must both be given or both be NULL");
    if (mask && words < 1) return fail(TOM_ERR_INVALID_ARG, "words = %d must be >= 1 with a mask", words);
    if ((reinterpret_cast<uintptr_t>(mask) & 7u) != 0) return fail(TOM_ERR_INVALID_ARG, "mask must be 8-byte aligned");
    if (!is_number(scale)) return fail(TOM_ERR_INVALID_ARG, "scale must be a number");
    if (!is_number(softcap) || softcap < 0.0f) return fail(TOM_ERR_INVALID_ARG, "softcap must be a number >= 0");
    if (!pages->starts && tokens != pages->sequences)
        return fail(TOM_ERR_INVALID_ARG, "%d tokens of %d sequences: without starts each has one", tokens, pages->sequences);
    if (tokens > kMaxNewTokens) return fail(TOM_ERR_UNSUPPORTED, "%d new tokens: at most %d per call", tokens, kMaxNewTokens);
    if ((int64_t)n_q_heads * tokens >= 1 << 30) return fail(TOM_ERR_UNSUPPORTED, "%d heads of %d tokens: less than 2^30 together per call", n_q_heads, tokens);
    if (tokens == 0 || pages->sequences == 0) return TOM_OK;
    if (tom_status_t st = check_view(q, "q", n_q_heads, tokens, channels, pages->dtype, 16, 1, a.q_head, a.q_row)) return st;
    if (tom_status_t st = check_view(out, "out", n_q_heads, tokens, channels, pages->dtype, 16, 1, a.out_head, a.out_row)) return st;
    if (!elements_apart(*out)) return fail(TOM_ERR_INVALID_ARG, "heads or rows of out overlap");
    if (prior_out) {
        if (tom_status_t st = check_view(prior_out, "prior_out", n_q_heads, tokens, channels, pages->dtype, 16, 1, a.prior_head, a.prior_row)) return st;
        if (tom_status_t st = check_view(prior_lse, "prior_lse", n_q_heads, tokens, 1, TOM_F32, 4, 4, a.prior_lse_head, a.prior_lse_row)) return st;
        a.prior_out = static_cast<const char*>(prior_out->data);
        a.prior_lse = static_cast<const float*>(prior_lse->data);
    }
    if (lse) {
        if (tom_status_t st = check_view(lse, "lse", n_q_heads, tokens, 1, TOM_F32, 4, 4, a.lse_head, a.lse_row)) return st;
        if (!elements_apart(*lse)) return fail(TOM_ERR_INVALID_ARG, "heads or rows of lse overlap");
        a.lse = static_cast<float*>(lse->data);
    }
    const PagesForm form = pages_form(*pages, tokens, n_q_heads);
    const PagesCuts cuts = pages_cuts(*pages, tokens, n_q_heads, form);
    const PagesWorkspace need = workspace_of(*pages, form, cuts);
    if ((uint64_t)cuts.items * (uint64_t)pages->heads * (form.block_rows == 256 || form.split ? 2 * kBlock : kBlock) > kMaxLanes)
        return fail(TOM_ERR_UNSUPPORTED, "%d heads of %d tokens need more lanes than the 2^32 - 1 of a launch", n_q_heads, tokens);
    if (need.all() > 0) {
        if (!workspace || workspace_bytes < need.all())
            return fail(TOM_ERR_INVALID_ARG, "workspace of %zu bytes needed, %zu given", need.all(), workspace_bytes);
        if ((reinterpret_cast<uintptr_t>(workspace) & 15u) != 0) return fail(TOM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
        char* const w = static_cast<char*>(workspace);
        a.part_out = reinterpret_cast<float*>(w);
        a.part_stat = reinterpret_cast<f32pair*>(w + need.out);
        a.unit_first = reinterpret_cast<uint32_t*>(w + need.out + need.stat);
    }
    a.p.tokens = tokens;
    a.k = static_cast<const char*>(pages->k) + layer_bytes(*pages, layer);
    a.v = static_cast<const char*>(pages->v) + layer_bytes(*pages, layer);
    a.q = static_cast<const char*>(q->data);
    a.out = static_cast<char*>(out->data);
    a.mask = reinterpret_cast<const uint64_t*>(mask);
    a.words = words;
    a.causal = causal != 0;
    a.channels = channels;
    a.kv_heads = pages->heads;
    a.inv_kv_heads = reciprocal_u32((uint32_t)a.kv_heads);
    a.repeat = n_q_heads / pages->heads;
    a.inv_repeat = reciprocal_u32((uint32_t)a.repeat);
    a.items = cuts.items;
    a.extra = cuts.extra;
    a.least = form.least;
    a.sorted = cuts.extra == 0 && pages->sequences <= kMostSorted && cuts.items * (uint64_t)pages->heads > 256;
    // Under a cap below 2^-30 all scores are zero to float32's last place beside the one of exp(0); one above 2^40 changes none of up to 2^28.
    if (softcap > 0.0f && softcap < 0x1p-30f) scale = softcap = 0.0f;
    if (softcap > 0x1p40f) softcap = 0.0f;
    if (std::fabs(softcap > 0.0f ? scale / softcap : scale) >= 0x1p50f)
        return fail(TOM_ERR_INVALID_ARG, "scale, or scale / softcap, must be below 2^50");
    constexpr float kLog2e = 1.4426950408889634f;
    a.scale_log2 = softcap > 0.0f ? 2.0f * kLog2e * scale / softcap : scale * kLog2e;
    a.cap_log2 = softcap * kLog2e;
    a.by_terms = std::fabs(a.scale_log2) >= 0x1p-16f && std::fabs(a.scale_log2) <= 0x1p12f;
    (void)hipGetLastError();  // an error that an earlier call of the process left behind is not this launch's
    const hipError_t err = launch_attend_pages(a, form, pages->dtype, static_cast<hipStream_t>(hip_stream));
    if (err != hipSuccess) return fail(TOM_ERR_HIP, "attend_pages launch: %s", hipGetErrorString(err));
    return TOM_OK;
}

}  // extern "C"
