// Trees, rows appended and rows kept, run on the host lane by lane (lanes/hip/hip_runtime.h) with arrays of exactly the documented sizes under AddressSanitizer:
// numbers on the device that make no sense lead to no address outside, and what makes sense comes out right.  Built by tests/test_pages_lanes.py.  Exit status 0 =
// clean.
#include <algorithm>
#include <cstdarg>
#include <random>

#include "oqm_append_rows.hip"
#include "oqm_draft.hip"

namespace oqm {
tom_status_t fail(tom_status_t st, const char*, ...) { return st; }
}  // namespace oqm

using namespace oqm;

static int failures = 0, calls = 0;
#define CHECK(x)                                                          \
    do {                                                                  \
        if (!(x)) {                                                       \
            std::fprintf(stderr, "line %d: %s is false\n", __LINE__, #x); \
            ++failures;                                                   \
        }                                                                 \
    } while (0)

template <typename T>
static T* exactly(size_t n, int byte = 0) {
    void* p = nullptr;
    if (posix_memalign(&p, 64, n * sizeof(T) ? n * sizeof(T) : 1)) std::abort();
    std::memset(p, byte, n * sizeof(T));
    return static_cast<T*>(p);
}
static std::mt19937 rng(11);
static int below(int n) { return (int)(rng() % (uint32_t)n); }

// Starts of one kind of nonsense; 0: as they should be.
static void set_starts(int32_t* starts, const std::vector<int>& news, int wrong) {
    const int B = (int)news.size();
    int T = 0;
    for (int n : news) T += n;
    for (int s = 0, at = 0; s <= B; ++s) {
        starts[s] = at;
        if (s < B) at += news[s];
        if (wrong == 1) starts[s] = s % 2 ? T : 0;
        if (wrong == 2) starts[s] = s % 2 ? 0 : T;
        if (wrong == 3) starts[s] = s ? T - s + 1 : -5;
        if (wrong == 4) starts[s] = (int32_t)rng();
        if (wrong == 5) starts[s] = below(T + 1);
        if (wrong == 6) starts[s] = s ? INT32_MAX : INT32_MIN;
    }
}

static void trees() {
    for (const std::vector<int>& news : {std::vector<int>{1}, {13}, {300}, {3, 0, 200, 1, 64}, {70, 1, 130}, {4200, 3}})
        for (int words : {1, 2, 64})
            for (int wrong = 0; wrong < 7; ++wrong) {
                const int B = (int)news.size();
                int T = 0;
                for (int n : news) T += n;
                if (T > 1000 && wrong > 1) continue;
                int32_t *starts = exactly<int32_t>(B + 1), *parents = exactly<int32_t>(T);
                int64_t *mask = exactly<int64_t>((size_t)T * words, 7), *first = exactly<int64_t>(B), *positions = exactly<int64_t>(T, 7);
                for (int t = 0; t < T; ++t) parents[t] = below(5) == 0 ? (int32_t)rng() : below(3) ? below(2 * T) - T / 2 : below(300) - 2;
                set_starts(starts, news, wrong);
                CHECK(tom_oqm_draft_tree(parents, starts, B, T, mask, words, first, positions, nullptr) == TOM_OK);
                ++calls;
                for (int s = 0; s < B && wrong == 0; ++s)
                    for (int j = 0; j < news[s]; ++j) {
                        std::vector<uint64_t> bits(words, 0);
                        int seen = 0;
                        for (int at = j; at >= 0;) {
                            if (at < 64 * words) bits[at / 64] |= uint64_t{1} << (at % 64);
                            ++seen;
                            const int p = parents[starts[s] + at];
                            at = p >= 0 && p < at ? p : -1;
                        }
                        const int64_t t = starts[s] + j;
                        CHECK(positions[t] == seen - 1 && std::memcmp(&mask[t * words], bits.data(), 8u * words) == 0);
                    }
                std::free(starts), std::free(parents), std::free(mask), std::free(first), std::free(positions);
            }
}

struct Pool {
    tom_oqm_pages_t g{};
    int32_t *table, *rows, *starts;
    int T = 0, width = 1, n_pages = 2, e;
    size_t bytes;
    std::vector<int> had, news;
    Pool(int layers, int heads, int channels, int dtype, std::vector<int> had_, std::vector<int> news_) : had(had_), news(news_) {
        const int B = (int)had.size(), P = 8;
        e = bytes_of_dtype(dtype);
        for (int s = 0; s < B; ++s) {
            const int used = (had[s] + news[s] + P - 1) / P;
            n_pages += used;
            width = std::max(width, used);
            T += news[s];
        }
        table = exactly<int32_t>((size_t)B * width);
        rows = exactly<int32_t>(B);
        starts = exactly<int32_t>(B + 1);
        const size_t pool = (size_t)layers * n_pages * heads * P * channels;
        bytes = pool * e;
        g.k = exactly<char>(bytes);
        g.v = exactly<char>(bytes);
        g.row_stride = channels;
        g.head_stride = (int64_t)P * channels;
        g.page_stride = heads * g.head_stride;
        g.layer_stride = n_pages * g.page_stride;
        g.n_layers = layers;
        g.n_pages = n_pages;
        g.heads = heads;
        g.page_rows = P;
        g.channels = channels;
        g.dtype = dtype;
        g.table = table;
        g.rows = rows;
        g.starts = starts;
        g.sequences = B;
        g.table_pages = width;
    }
    ~Pool() { std::free(g.k), std::free(g.v), std::free(table), std::free(rows), std::free(starts); }
    void set(int wrong) {
        const int B = (int)had.size(), P = 8;
        set_starts(starts, news, wrong);
        for (int s = 0, at = 1; s < B; ++s) {
            rows[s] = wrong == 7 ? (int32_t)rng() : wrong == 8 ? (s % 2 ? INT32_MAX : width * P) : had[s];
            for (int i = 0; i < width; ++i) {
                table[s * width + i] = i < (had[s] + news[s] + P - 1) / P ? at++ : -1;
                if (wrong == 9 && below(2)) table[s * width + i] = below(3) ? (int32_t)rng() : n_pages;
            }
        }
        for (size_t i = 0; i < bytes; ++i) {
            static_cast<uint8_t*>(g.k)[i] = (uint8_t)(i * 7 + i / 251);
            static_cast<uint8_t*>(g.v)[i] = (uint8_t)(i * 5 + i / 241);
        }
    }
    char* row(void* base, int layer, int s, int head, int r) const {
        return static_cast<char*>(base) + ((int64_t)layer * g.layer_stride + table[s * width + r / 8] * g.page_stride + head * g.head_stride + (r % 8) * g.row_stride) * e;
    }
};

static void kept() {
    for (int dtype : {(int)TOM_BF16, (int)TOM_F32})
        for (const auto& [had, news] : {std::pair<std::vector<int>, std::vector<int>>{{20}, {13}}, {{7, 0, 30}, {5, 1, 40}}, {{3, 3, 3, 3}, {300, 0, 20, 2}}})
            for (int channels : {8, 72})
                for (int wrong = 0; wrong < 12; ++wrong) {
                    Pool p(2, 2, channels, dtype, had, news);
                    const int B = (int)had.size(), width = 12;
                    p.set(wrong);
                    int32_t *idx = exactly<int32_t>((size_t)B * width), *counts = exactly<int32_t>(B), *out = exactly<int32_t>(B);
                    for (int s = 0; s < B; ++s) {
                        counts[s] = std::min({width, news[s], 1 + below(width)});
                        std::vector<int> all(news[s]);
                        for (int i = 0; i < news[s]; ++i) all[i] = i;
                        std::shuffle(all.begin(), all.end(), rng);
                        std::sort(all.begin(), all.begin() + counts[s]);
                        for (int i = 0; i < width; ++i) idx[s * width + i] = i < counts[s] ? all[i] : (int32_t)rng();
                        if (wrong == 10) counts[s] = (int32_t)rng();
                        for (int i = 0; i < width && wrong == 11; ++i) idx[s * width + i] = below(2) ? (int32_t)rng() : below(60) - 3;
                    }
                    std::vector<char> k(static_cast<char*>(p.g.k), static_cast<char*>(p.g.k) + p.bytes), v(static_cast<char*>(p.g.v), static_cast<char*>(p.g.v) + p.bytes);
                    CHECK(tom_oqm_keep_rows(&p.g, idx, width, counts, wrong % 2 ? p.rows : out, nullptr) == TOM_OK);
                    ++calls;
                    for (int s = 0; s < B && wrong == 0; ++s) {
                        CHECK(out[s] == had[s] + counts[s]);
                        for (int i = 0; i < counts[s]; ++i)
                            for (int layer = 0; layer < 2; ++layer)
                                for (int head = 0; head < 2; ++head) {
                                    const size_t from = p.row(p.g.k, layer, s, head, had[s] + idx[s * width + i]) - static_cast<char*>(p.g.k), n = (size_t)channels * p.e;
                                    CHECK(!std::memcmp(p.row(p.g.k, layer, s, head, had[s] + i), &k[from], n) && !std::memcmp(p.row(p.g.v, layer, s, head, had[s] + i), &v[from], n));
                                }
                    }
                    std::free(idx), std::free(counts), std::free(out);
                }
}

static void appended() {
    struct Size {
        int channels, rotary_dim, layout, dtype, offset;  // offset: elements in front of the first, so that lanes take single elements
    };
    for (const Size& z : {Size{64, 64, TOM_ROTARY_HALF, TOM_BF16, 0}, Size{72, 30, TOM_ROTARY_PAIRS, TOM_BF16, 0}, Size{256, 256, TOM_ROTARY_HALF, TOM_F32, 1}, Size{8, 2, TOM_ROTARY_PAIRS, TOM_F32, 0}})
        for (const auto& [had, news] : {std::pair<std::vector<int>, std::vector<int>>{{20}, {13}}, {{7, 0, 30, 3}, {5, 1, 20, 0}}})
            for (int wrong = 0; wrong < 10; ++wrong) {
                Pool p(2, 2, z.channels, z.dtype, had, news);
                p.set(wrong);
                const int B = (int)had.size(), T = p.T, q_heads = 4, per = (q_heads + 4) * z.channels;
                tom_oqm_rotary_t rotary{};
                rotary.rotary_dim = z.rotary_dim;
                rotary.layout = z.layout;
                rotary.original_length = 1;
                rotary.base = 10000.0;
                rotary.factor = 1.0;
                double* const turns = exactly<double>(z.rotary_dim / 2);
                int64_t* const positions = exactly<int64_t>(T);
                char* const x = exactly<char>(((size_t)T * per + z.offset) * p.e, 0x31);
                char* const out = exactly<char>((size_t)T * q_heads * z.channels * p.e);
                for (size_t i = 0; i < (size_t)T * per; ++i) x[(i + z.offset) * p.e] = (char)(i * 3);
                char* const norm = exactly<char>((size_t)z.channels * p.e, 0x3f);
                auto view = [&](int head, int heads) {
                    tom_oqm_view_t v{};
                    v.data = x + ((size_t)z.offset + (size_t)head * z.channels) * p.e;
                    v.heads = heads;
                    v.rows = T;
                    v.channels = z.channels;
                    v.dtype = z.dtype;
                    v.head_stride = z.channels;
                    v.row_stride = per;
                    return v;
                };
                const tom_oqm_view_t q = view(0, q_heads), k = view(q_heads, 2), v = view(q_heads + 2, 2);
                tom_oqm_view_t q_out = q;
                q_out.data = out;
                q_out.row_stride = q_heads * z.channels;
                CHECK(tom_oqm_append_rows(&p.g, 1, &rotary, turns, 1.0f, positions, &q, &q_out, &k, &v, wrong % 3 ? norm : nullptr, norm, 1e-6f, nullptr) == TOM_OK);
                ++calls;
                for (int s = 0, t = 0; s < B && wrong == 0; ++s)
                    for (int j = 0; j < news[s]; ++j, ++t)
                        for (int head = 0; head < 2; ++head)
                            CHECK(!std::memcmp(p.row(p.g.v, 1, s, head, had[s] + j), static_cast<char*>(v.data) + ((size_t)t * per + (size_t)head * z.channels) * p.e, (size_t)z.channels * p.e));
                std::free(turns), std::free(positions), std::free(x), std::free(out), std::free(norm);
            }
}

template <typename T, int V, bool PAIRS>
static void rotates() {
    lanes::runs(rotate_kernel<T, V, PAIRS, true, false, AppendArgs>);
    lanes::runs(rotate_kernel<T, V, PAIRS, false, false, AppendArgs>);
    if constexpr (V * elem_bytes<T>::value == 16) lanes::runs(rotate_kernel<T, V, PAIRS, false, true, AppendArgs>);
    if constexpr (V > 1) rotates<T, V / 2, PAIRS>();
}

int main() {
    lanes::runs(draft_tree_kernel);
    lanes::runs(keep_rows_kernel);
    lanes::runs(kept_rows_kernel);
    rotates<In_f32, 4, false>();
    rotates<In_f32, 4, true>();
    rotates<In_bf16, 8, false>();
    rotates<In_bf16, 8, true>();
    trees();
    kept();
    appended();
    CHECK(calls > 300);
    if (failures) return 1;
    std::printf("rows lanes driver: clean, %d calls\n", calls);
    return 0;
}
