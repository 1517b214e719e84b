// New rows of several sequences: queries and keys normed and turned as tom_oqm_rotate does, keys and values written to the pages of
// their sequences.  The kernel is the rotary's, with one more step in front: whose token it is, and where its row lies.
#include "oqm_rotate.h"

using namespace oqm;

extern "C" {

tom_status_t tom_oqm_append_rows(const tom_oqm_pages_t* pages, int32_t layer, const tom_oqm_rotary_t* r, const double* turns, float amplitude,
                                 const int64_t* positions, const tom_oqm_view_t* q, const tom_oqm_view_t* q_out, const tom_oqm_view_t* k,
                                 const tom_oqm_view_t* v, const void* q_norm, const void* k_norm, float norm_eps, void* hip_stream) {
    if (tom_status_t st = check_rotary(r)) return st;
    AppendArgs g{};
    if (tom_status_t st = check_pages(pages, g.pages)) return st;
    if (layer < 0 || layer >= pages->n_layers) return fail(TOM_ERR_INVALID_ARG, "layer %d is outside [0, %d)", layer, pages->n_layers);
    if (!k || !v) return fail(TOM_ERR_INVALID_ARG, "k and v must be non-NULL");
    if (!q != !q_out) return fail(TOM_ERR_INVALID_ARG, "q and its output must both be given or both be NULL");
    if (q_norm && !q) return fail(TOM_ERR_INVALID_ARG, "norm weights are given for q, which is not");
    constexpr int64_t kMaxStride = int64_t{1} << 40;  // elements; far beyond any device tensor
    const tom_oqm_view_t* const in[4] = {q, k, v, q_out};
    static const char* const name[4] = {"q", "k", "v", "q_out"};
    for (int i = 0; i < 4; ++i) {
        const tom_oqm_view_t* t = in[i];
        if (!t) continue;
        if (t->heads < 0 || t->rows < 0) return fail(TOM_ERR_INVALID_ARG, "%s has a negative size", name[i]);
        if (t->dtype != pages->dtype || t->rows != k->rows || t->channels != pages->channels)
            return fail(TOM_ERR_INVALID_ARG, "%s must have the pages' dtype and channels, and k's rows", name[i]);
        if (t->heads != (i == 0 || i == 3 ? q->heads : pages->heads))
            return fail(TOM_ERR_INVALID_ARG, "k and v must have the pages' heads, and q_out q's");
        if (t->head_stride < 0 || t->row_stride < 0 || t->head_stride > kMaxStride || t->row_stride > kMaxStride)
            return fail(TOM_ERR_INVALID_ARG, "strides of %s must be in [0, 2^40] elements", name[i]);
    }
    if (q_out && !elements_apart(*q_out)) return fail(TOM_ERR_INVALID_ARG, "heads or rows of q_out overlap");
    const int32_t tokens = k->rows, channels = pages->channels;
    if (channels < r->rotary_dim) return fail(TOM_ERR_INVALID_ARG, "channels = %d must be at least rotary_dim = %d", channels, r->rotary_dim);
    if (!is_number(norm_eps) || norm_eps < 0.0f) return fail(TOM_ERR_INVALID_ARG, "norm_eps must be a number >= 0");
    if (!is_number(amplitude)) return fail(TOM_ERR_INVALID_ARG, "amplitude must be a number");
    if (!pages->starts && tokens != pages->sequences)
        return fail(TOM_ERR_INVALID_ARG, "%d tokens of %d sequences: without starts each has one", tokens, pages->sequences);
    if (tokens == 0 || pages->sequences == 0) return TOM_OK;
    const int e = bytes_of_dtype(pages->dtype);
    uintptr_t low_bits = 0;  // of every address and byte stride
    int64_t heads = 0;
    for (int i = 0; i < 3; ++i) {
        RotateSide& d = g.side[i];
        if (!in[i] || in[i]->heads == 0) continue;
        if (!in[i]->data || (i == 0 && !q_out->data)) return fail(TOM_ERR_INVALID_ARG, "%s and its output must have data", name[i]);
        d.in = static_cast<const char*>(in[i]->data);
        d.in_head = in[i]->heads > 1 ? in[i]->head_stride * e : 0;
        d.in_row = tokens > 1 ? in[i]->row_stride * e : 0;
        if (i == 0) {
            d.out = static_cast<char*>(q_out->data);
            d.out_head = q->heads > 1 ? q_out->head_stride * e : 0;
            d.out_row = tokens > 1 ? q_out->row_stride * e : 0;
        } else {
            d.out = static_cast<char*>(i == 1 ? pages->k : pages->v) + layer_bytes(*pages, layer);
            d.out_head = g.pages.head_bytes;
        }
        d.norm = static_cast<const char*>(i == 0 ? q_norm : i == 1 ? k_norm : nullptr);
        d.heads = in[i]->heads;
        d.turned = i < 2;
        heads += d.heads;
        low_bits |= reinterpret_cast<uintptr_t>(d.in) | reinterpret_cast<uintptr_t>(d.out) | reinterpret_cast<uintptr_t>(d.norm) |
                    (uintptr_t)d.in_head | (uintptr_t)d.in_row | (uintptr_t)d.out_head | (uintptr_t)d.out_row;
    }
    if (low_bits % e) return fail(TOM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    if (!turns || !positions) return fail(TOM_ERR_INVALID_ARG, "turns and positions must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(turns) | reinterpret_cast<uintptr_t>(positions)) & 7u)
        return fail(TOM_ERR_INVALID_ARG, "turns and positions must be 8-byte aligned");
    if ((uint64_t)tokens * (uint64_t)heads > 0x7fffffffu)
        return fail(TOM_ERR_UNSUPPORTED, "rows * heads exceeds 2^31 - 1: append fewer rows per call");
    g.pages.tokens = tokens;
    return launch_rotate(g, r, "append_rows", pages->dtype, tokens, channels, heads, low_bits, k->row_stride < k->head_stride, amplitude, norm_eps, turns, positions,
                         hip_stream);
}

}  // extern "C"
