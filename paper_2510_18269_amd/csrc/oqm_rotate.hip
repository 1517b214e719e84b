// Rotary positions of new queries and keys, after a norm of every head where asked, and the copy of their values: one launch
// between a projection and the cache.
//
//   x' = x * w / sqrt(mean(x^2) + eps)                 (a, b) -> A (a cos t - b sin t, b cos t + a sin t), t = position * turns
//
// Every element is read once and written once, so memory bounds large calls and the launch small ones.  The cosines are the only
// arithmetic of weight: one float64 product and reduction a (token, pair), which the heads of a token share.
#include <cmath>

#include "oqm_rotate.h"

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
    const int e = bytes_of_dtype(one->dtype);
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

    return launch_rotate(g, r, "rotate", one->dtype, one->rows, one->channels, heads, low_bits, one->row_stride < one->head_stride, amplitude, norm_eps, turns,
                         positions, hip_stream);
}

}  // extern "C"
