// Sanitizer driver for the host side of the calls on pages and for the rules that cut the attention over them: built for the host with
// -fsanitize=address,undefined by tests/test_sanitizers_pages.py.  The launchers of the attention are stubs that count; device pointers are fakes, and every
// other call below is refused or a documented no-op.  Exit status 0 = clean.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "oqm_attend_pages.h"

namespace oqm {
#define STUB(name, ...) \
    hipError_t name(__VA_ARGS__) { std::abort(); }
STUB(launch_quantize_append, const QuantArgs&, int, hipStream_t)
STUB(launch_dequant_gather, const DequantArgs&, int, hipStream_t)
STUB(launch_prefix_copy, const DequantArgs&, const void*, const void*, int, hipStream_t)
STUB(launch_score_mean_query, const ScoreArgs&, hipStream_t)
STUB(launch_score_token_gemm, const ScoreArgs&, hipStream_t)
STUB(launch_topk, const float*, int64_t, int, int, int, int, int, int32_t*, hipStream_t)
static int launched = 0;
void start_attend_pages_f32(const PagesArgs&, const PagesForm&, hipStream_t) { ++launched; }
void start_attend_pages_bf16(const PagesArgs&, const PagesForm&, hipStream_t) { ++launched; }
void start_attend_pages_f16(const PagesArgs&, const PagesForm&, hipStream_t) { ++launched; }
}  // namespace oqm

using namespace oqm;

static int failures = 0;
#define CHECK(x)                                                          \
    do {                                                                  \
        if (!(x)) {                                                       \
            std::fprintf(stderr, "line %d: %s is false\n", __LINE__, #x); \
            ++failures;                                                   \
        }                                                                 \
    } while (0)

static tom_oqm_pages_t some_pages(int32_t heads, int32_t channels, int32_t dtype, int32_t sequences, int32_t table_pages, int32_t page_rows, const int32_t* starts) {
    tom_oqm_pages_t g{};
    g.k = reinterpret_cast<void*>(uintptr_t{0x100000});
    g.v = reinterpret_cast<void*>(uintptr_t{0x200000});
    g.row_stride = channels;
    g.head_stride = (int64_t)page_rows * channels;
    g.page_stride = heads * g.head_stride;
    g.n_pages = 3;
    g.layer_stride = g.n_pages * g.page_stride;
    g.n_layers = 2;
    g.heads = heads;
    g.page_rows = page_rows;
    g.channels = channels;
    g.dtype = dtype;
    g.table = g.rows = reinterpret_cast<const int32_t*>(uintptr_t{0x300000});
    g.starts = starts;
    g.sequences = sequences;
    g.table_pages = table_pages;
    return g;
}

// What the workgroups work out on the device from rows and starts: that the launch has one for every part of every block, whatever the lengths are.
static void parts_have_workgroups() {
    std::mt19937 rng(1);
    auto below = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)n); };
    const int32_t* const some = reinterpret_cast<const int32_t*>(uintptr_t{0x400000});
    for (int round = 0; round < 4000; ++round) {
        const int32_t heads = 1 + (int32_t)below(9), repeat = 1 + (int32_t)below(20), sequences = 1 + (int32_t)below(round % 3 ? 12 : 600);
        const int32_t channels = 8 * (1 + (int32_t)below(32)), page_rows = 1 + (int32_t)below(300), table_pages = (int32_t)below(round % 2 ? 2000 : 20);
        std::vector<int32_t> news(sequences), rows(sequences);
        const int64_t most = 1 + below(round % 5 ? 9 : 400);
        int64_t tokens = 0;
        for (int32_t s = 0; s < sequences; ++s) {
            news[s] = (int32_t)below(most + 1);
            rows[s] = (int32_t)below((int64_t)table_pages * page_rows + 1);
            tokens += news[s];
        }
        if (tokens == 0 || tokens * heads * repeat >= 1 << 30) continue;
        const tom_oqm_pages_t g = some_pages(heads, channels, (int32_t)(round % 3 == 0 ? TOM_F32 : round % 3 == 1 ? TOM_BF16 : TOM_F16), sequences, table_pages, page_rows, some);
        const PagesForm f = pages_form(g, (int32_t)tokens, heads * repeat);
        const PagesCuts c = pages_cuts(g, (int32_t)tokens, heads * repeat, f);
        const int64_t capacity = (int64_t)table_pages * page_rows;
        for (int64_t tile : {32, 64}) {
            int64_t total = 0, items = 0;
            for (int32_t s = 0; s < sequences; ++s) {
                const int64_t tiles = ((int64_t)news[s] * repeat + f.block_rows - 1) / f.block_rows, all = std::min(capacity, (int64_t)rows[s] + news[s]);
                total += tiles * all;
            }
            const int64_t chunk = c.extra ? std::max((total / c.extra + tile) / tile * tile, (int64_t)f.least) : INT64_MAX / 4;
            for (int32_t s = 0; s < sequences; ++s) {
                const int64_t tiles = ((int64_t)news[s] * repeat + f.block_rows - 1) / f.block_rows, all = std::min(capacity, (int64_t)rows[s] + news[s]);
                items += tiles * std::max((all + chunk - 1) / chunk, (int64_t)1);
            }
            CHECK(items <= (int64_t)c.items);
        }
        // a block's place in the list of units: unlike every other's, and inside
        int64_t first = 0, last = -1;
        for (int32_t s = 0; s < sequences; ++s) {
            const int64_t tiles = ((int64_t)news[s] * repeat + f.block_rows - 1) / f.block_rows;
            const int64_t unit = first * repeat / f.block_rows + std::min<int64_t>(s, first);
            if (tiles > 0) {
                CHECK(unit > last);
                last = unit + tiles - 1;
                CHECK(last < (int64_t)c.units);
            }
            first += news[s];
        }
        CHECK(c.extra == 0 || (tom_oqm_attend_pages_workspace_bytes(&g, (int32_t)tokens, heads * repeat) >= (size_t)c.items * heads * f.block_rows * (channels * 4u + 8u)));
    }
}

// Every number of a call at its ends: refused, or launched with what the checks have let through.
static void odd_numbers() {
    const int32_t* const some = reinterpret_cast<const int32_t*>(uintptr_t{0x400000});
    const int32_t values[] = {INT32_MIN, -1, 0, 1, 7, 8, 64, 256, 65536, (1 << 20) + 1, INT32_MAX};
    const int64_t strides[] = {INT64_MIN, -16, 0, 8, 64, int64_t{1} << 40, (int64_t{1} << 40) + 16, INT64_MAX};
    void* const fake = reinterpret_cast<void*>(uintptr_t{0x500000});
    auto call = [&](const tom_oqm_pages_t& g, int32_t tokens, int32_t heads, float scale, float cap) {
        tom_oqm_view_t q{};
        q.data = fake;
        q.channels = g.channels;
        q.rows = tokens;
        q.heads = heads;
        q.dtype = g.dtype;
        q.row_stride = (int64_t)heads * g.channels;
        q.head_stride = g.channels;
        (void)tom_oqm_attend_pages_workspace_bytes(&g, tokens, heads);
        (void)tom_oqm_attend_pages(&g, 0, &q, &q, nullptr, 0, 1, scale, cap, nullptr, nullptr, nullptr, fake, SIZE_MAX / 2, nullptr);
        (void)tom_oqm_keep_rows(&g, nullptr, -1, some, nullptr, nullptr);
        (void)tom_oqm_draft_tree(nullptr, some, g.sequences, tokens, nullptr, 1, nullptr, nullptr, nullptr);
    };
    for (int32_t v : values) {
        for (int field = 0; field < 8; ++field) {
            tom_oqm_pages_t g = some_pages(2, 64, TOM_BF16, 4, 50, 16, some);
            int32_t* const at[8] = {&g.n_layers, &g.n_pages, &g.heads, &g.page_rows, &g.channels, &g.dtype, &g.sequences, &g.table_pages};
            *at[field] = v;
            call(g, 7, 6, 0.1f, 0.0f);
        }
        const tom_oqm_pages_t g = some_pages(2, 64, TOM_BF16, 4, 50, 16, some);
        call(g, v, 6, 0.1f, 0.0f);
        call(g, 7, v, 0.1f, 0.0f);
    }
    for (int64_t v : strides)
        for (int field = 0; field < 4; ++field) {
            tom_oqm_pages_t g = some_pages(2, 64, TOM_F32, 4, 50, 16, some);
            int64_t* const at[4] = {&g.layer_stride, &g.page_stride, &g.head_stride, &g.row_stride};
            *at[field] = v;
            call(g, 7, 6, 0.1f, 0.0f);
        }
    const float numbers[] = {0.0f, -0.0f, 1.0f, -3.0f, 1e-38f, 1e38f, INFINITY, -INFINITY, NAN};
    for (float scale : numbers)
        for (float cap : numbers) call(some_pages(2, 64, TOM_F16, 4, 50, 16, some), 7, 6, scale, cap);
    CHECK(launched > 0);
}

int main() {
    parts_have_workgroups();
    odd_numbers();
    if (failures) return 1;
    std::printf("pages driver: clean\n");
    return 0;
}
