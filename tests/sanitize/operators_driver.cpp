// Sanitizer driver for the host side of the rotary, the attention over stored groups and the moves of groups: built for the host
// with -fsanitize=address,undefined by tests/test_sanitizers_operators.py.  Every call below is refused by the validation or a
// documented no-op; the attention's launcher is a stub that aborts, device pointers are fakes.  Exit status 0 = clean.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "oqm_attend.h"

namespace oqm {
#define STUB(name, ...)                                                                                  \
    hipError_t name(__VA_ARGS__) {                                                                       \
        std::fprintf(stderr, "launcher " #name " reached: validation let a bad call through\n");         \
        std::abort();                                                                                    \
    }
STUB(launch_quantize_append, const QuantArgs&, int, hipStream_t)
STUB(launch_dequant_gather, const DequantArgs&, int, hipStream_t)
STUB(launch_prefix_copy, const DequantArgs&, const void*, const void*, int, hipStream_t)
STUB(launch_score_mean_query, const ScoreArgs&, hipStream_t)
STUB(launch_score_token_gemm, const ScoreArgs&, hipStream_t)
STUB(launch_topk, const float*, int64_t, int, int, int, int, int, int32_t*, hipStream_t)
STUB(launch_attend, const AttendArgs&, const AttendForm&, int, hipStream_t)
}  // namespace oqm

static int failures = 0;
#define EXPECT(call, want)                                                                                                   \
    do {                                                                                                                     \
        const int got_ = (int)(call);                                                                                        \
        if (got_ != (int)(want)) {                                                                                           \
            std::fprintf(stderr, "line %d: %s -> %d (%s), wanted %d\n", __LINE__, #call, got_, tom_last_error(), (int)(want)); \
            ++failures;                                                                                                      \
        }                                                                                                                    \
    } while (0)

int main() {
    void* const fake = reinterpret_cast<void*>(uintptr_t{0x10000});
    int32_t* const idx = static_cast<int32_t*>(fake);
    const int32_t odd_values[] = {INT32_MIN, -1, 0, 1, 3, 7, 100, 65536, INT32_MAX};

    // rotary: every field at odd values; what is accepted fills its whole array and stays finite
    tom_oqm_rotary_t good = {64, TOM_ROTARY_HALF, TOM_ROTARY_PLAIN, 4096, 10000.0, 4.0};
    float amplitude = 0;
    std::vector<double> turns(1024);
    EXPECT(tom_oqm_rotary_turns(nullptr, turns.data(), &amplitude), TOM_ERR_INVALID_ARG);
    EXPECT(tom_oqm_rotary_turns(&good, nullptr, &amplitude), TOM_ERR_INVALID_ARG);
    EXPECT(tom_oqm_rotary_turns(&good, turns.data(), nullptr), TOM_ERR_INVALID_ARG);
    for (int scaling = 0; scaling < 5; ++scaling)
        for (int n : {2, 4, 6, 64, 130, 2048})
            for (int32_t original : {1, 2, 4096, INT32_MAX})
                for (double base : {1.0000001, 10000.0, 1e30})
                    for (double factor : {1.0, 7.3, 1e6}) {
                        tom_oqm_rotary_t r = {n, 0, scaling, original, base, factor};
                        std::vector<double> own(n / 2, -1.0);
                        if (scaling == TOM_ROTARY_BASE && n < 4) {
                            EXPECT(tom_oqm_rotary_turns(&r, own.data(), &amplitude), TOM_ERR_INVALID_ARG);
                            continue;
                        }
                        EXPECT(tom_oqm_rotary_turns(&r, own.data(), &amplitude), TOM_OK);
                        for (double t : own)
                            if (!(t >= 0.0 && t <= 0.16)) ++failures;
                    }
    for (int field = 0; field < 4; ++field)
        for (int32_t v : odd_values) {
            tom_oqm_rotary_t r = good;
            reinterpret_cast<int32_t*>(&r)[field] = v;
            if (v == 100 && field == 0) continue;
            (void)tom_oqm_rotary_turns(&r, turns.data(), &amplitude);
        }
    auto view = [&](int heads, int rows, int channels, int dtype) {
        return tom_oqm_view_t{fake, (int64_t)channels * (rows > 0 ? rows : 1), channels, heads, rows, channels, dtype};
    };
    const double* const angles = static_cast<const double*>(fake);
    const int64_t* const at = static_cast<const int64_t*>(fake);
    const tom_oqm_view_t q = view(4, 3, 64, TOM_BF16);
    auto rotate = [&](const tom_oqm_view_t* in, const tom_oqm_view_t* out) {
        return tom_oqm_rotate(&good, angles, 1.0f, at, in, out, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 1e-6f, nullptr);
    };
    EXPECT(rotate(&q, nullptr), TOM_ERR_INVALID_ARG);
    EXPECT(rotate(nullptr, nullptr), TOM_OK);
    for (int field = 0; field < 4; ++field)
        for (int32_t v : odd_values) {  // heads, rows, channels, dtype of the output alone
            tom_oqm_view_t out = q;
            (&out.heads)[field] = v;
            if ((field == 1 && v == 3) || (field == 3 && v == TOM_BF16)) continue;
            EXPECT(rotate(&q, &out), TOM_ERR_INVALID_ARG);
        }
    for (int64_t stride : {int64_t{-1}, INT64_MIN, INT64_MAX, (int64_t{1} << 40) + 1}) {
        tom_oqm_view_t in = q;
        in.head_stride = stride;
        EXPECT(rotate(&in, &q), TOM_ERR_INVALID_ARG);
        in = q;
        in.row_stride = stride;
        EXPECT(rotate(&in, &q), TOM_ERR_INVALID_ARG);
    }
    tom_oqm_view_t huge = view(65536, 65536, 64, TOM_BF16);
    huge.head_stride = 64;
    huge.row_stride = int64_t{64} << 16;
    EXPECT(rotate(&huge, &huge), TOM_ERR_UNSUPPORTED);
    const tom_oqm_view_t none = view(0, 3, 64, TOM_BF16);
    EXPECT(rotate(&none, &none), TOM_OK);

    // attention
    tom_oqm_config_t cfg = {2, 2, 4, 64, 16, 32, TOM_QAXIS_HEAD_DIM, 4, 8, TOM_BF16, TOM_BF16, TOM_SIM_COSINE, TOM_F32};
    tom_oqm_t* h = nullptr;
    EXPECT(tom_oqm_create(&cfg, &h), TOM_OK);
    auto attend = [&](int32_t layer, const tom_oqm_view_t* in, const tom_oqm_view_t* out, int32_t k, const tom_oqm_view_t* rows, float scale = 1.0f,
                      float cap = 0.0f) {
        return tom_oqm_attend(h, layer, in, out, idx, k, nullptr, nullptr, rows, rows, 1, scale, cap, nullptr, nullptr, 0, nullptr);
    };
    const tom_oqm_view_t rows = view(2, 3, 64, TOM_BF16);
    EXPECT(attend(0, &q, &q, 4, nullptr), TOM_ERR_NOT_BOUND);
    EXPECT(tom_oqm_bind(h, fake, fake, fake), TOM_OK);
    for (int32_t layer : {INT32_MIN, -1, 2, INT32_MAX}) EXPECT(attend(layer, &q, &q, 0, nullptr), TOM_ERR_INVALID_ARG);
    for (int32_t k : {INT32_MIN, -1}) EXPECT(attend(0, &q, &q, k, nullptr), TOM_ERR_INVALID_ARG);
    EXPECT(attend(0, &q, &q, INT32_MAX, nullptr), TOM_ERR_UNSUPPORTED);
    EXPECT(attend(0, &q, &q, 1, &rows, NAN), TOM_ERR_INVALID_ARG);
    EXPECT(attend(0, &q, &q, 1, &rows, INFINITY), TOM_ERR_INVALID_ARG);
    EXPECT(attend(0, &q, &q, 1, &rows, 1.0f, NAN), TOM_ERR_INVALID_ARG);
    for (int field = 0; field < 4; ++field)
        for (int32_t v : odd_values) {
            if ((field == 1 && v == 3) || (field == 3 && v == TOM_BF16)) continue;
            tom_oqm_view_t out = q, r = rows;
            (&out.heads)[field] = v;
            EXPECT(attend(0, &q, &out, 0, nullptr), TOM_ERR_INVALID_ARG);
            (&r.heads)[field] = v;
            if (field == 1) r.rows = v < 0 ? v : -1;
            EXPECT(attend(0, &q, &q, 0, &r), TOM_ERR_INVALID_ARG);
        }
    for (int64_t stride : {int64_t{-8}, INT64_MIN, INT64_MAX / 8 * 8, int64_t{65}}) {
        tom_oqm_view_t r = rows;
        r.row_stride = stride;
        EXPECT(attend(0, &q, &q, 0, &r), TOM_ERR_INVALID_ARG);
    }
    // the cut of a call: at least one part, never fewer for more rows, a bounded workspace, all of it addressable in 64 bits
    for (int32_t H : {1, 4, 8, 128})
        for (int32_t R : {1, 7, 64})
            for (int32_t d : {8, 64, 128, 256})
                for (int32_t dtype : {TOM_F32, TOM_BF16})
                    for (int32_t axis : {0, 1})
                        for (int32_t t_q : {1, 2, 9, 64, 1000, 1 << 20}) {
                            tom_oqm_config_t c = {1, H, H * R, d, 50, 8, axis, 4, 8, dtype, dtype, 0, TOM_F32};
                            if (d >= 32) c.qgroup = 32;
                            const oqm::AttendForm form = oqm::attend_form(c, t_q);
                            if (form.rows != 16 && form.rows != 64 && form.rows != 128 && form.rows != 256) ++failures;
                            int32_t last = 0;
                            for (int64_t n : {int64_t{0}, int64_t{1}, int64_t{31}, int64_t{500}, int64_t{40000}, int64_t{1000000}, int64_t{2000000000}}) {
                                const int32_t cuts = oqm::attend_cuts(c, t_q, n);
                                if (cuts < 1 || cuts < last || (cuts > 1 && (int64_t)cuts * H * R * t_q > (int64_t)4096 * 16 * 64)) {
                                    std::fprintf(stderr, "H %d R %d d %d t_q %d n %lld: %d parts\n", H, R, d, t_q, (long long)n, cuts);
                                    ++failures;
                                }
                                last = cuts;
                            }
                        }

    // groups
    EXPECT(tom_oqm_set_num_groups(h, 5), TOM_OK);
    for (int32_t n : {INT32_MIN, -1, 6, INT32_MAX}) EXPECT(tom_oqm_keep_groups(h, idx, n, nullptr), TOM_ERR_INVALID_ARG);
    EXPECT(tom_oqm_keep_groups(h, nullptr, 1, nullptr), TOM_ERR_INVALID_ARG);
    EXPECT(tom_oqm_copy_groups(h, h, idx, INT32_MIN, nullptr), TOM_ERR_INVALID_ARG);
    EXPECT(tom_oqm_copy_groups(h, h, idx, 4, nullptr), TOM_ERR_CAPACITY);
    EXPECT(tom_oqm_copy_groups(h, h, idx, INT32_MAX, nullptr), TOM_ERR_CAPACITY);
    EXPECT(tom_oqm_copy_groups(h, nullptr, idx, 1, nullptr), TOM_ERR_INVALID_ARG);
    tom_oqm_t* other = nullptr;
    EXPECT(tom_oqm_create(&cfg, &other), TOM_OK);
    EXPECT(tom_oqm_copy_groups(other, h, idx, 1, nullptr), TOM_ERR_NOT_BOUND);
    EXPECT(tom_oqm_bind(other, fake, static_cast<char*>(fake) + 16, fake), TOM_OK);
    EXPECT(tom_oqm_copy_groups(other, h, idx, 1, nullptr), TOM_ERR_INVALID_ARG);
    EXPECT(tom_oqm_keep_groups(h, nullptr, 0, nullptr), TOM_OK);
    if (tom_oqm_num_groups(h) != 0) ++failures;
    tom_oqm_destroy(other);
    tom_oqm_destroy(h);
    if (failures) {
        std::fprintf(stderr, "%d failures\n", failures);
        return 2;
    }
    std::printf("operators sanitizer driver: clean\n");
    return 0;
}
