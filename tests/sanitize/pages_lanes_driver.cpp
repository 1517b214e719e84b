// The attention over pages, its kernel for few query rows and its joins, run on the host lane by lane (lanes/hip/hip_runtime.h) with arrays of exactly the documented
// sizes under AddressSanitizer: numbers on the device that make no sense, and sums that are none, are never trusted with an address.  Built by
// tests/test_pages_lanes.py.  Exit status 0 = clean.
#include "oqm_attend_pages_few.h"

#include <cstdarg>
#include <random>

namespace oqm {

tom_status_t fail(tom_status_t st, const char*, ...) { return st; }

static uint32_t most_extra = ~0u;  // further workgroups a call has here at most: those of a whole chip take long
static int blocks_run = 0;

template <typename F>
static void run(PagesArgs g) {
    if (g.extra > most_extra) {
        g.items -= g.extra - most_extra;
        g.extra = most_extra;
    }
    for (uint32_t x = 0; x < g.items * (uint32_t)g.kv_heads; ++x, ++blocks_run) {
        lanes::block_index = dim3(x);
        lanes::run_block(kBlock, [&] { attend_pages_few_kernel<F>(g); });
    }
    if (!g.extra) return;
    const uint32_t heads = (uint32_t)(g.kv_heads * g.repeat), rows = heads * (uint32_t)g.p.tokens, lanes_log2 = g.channels <= 64 ? 4 : g.channels <= 128 ? 5 : 6;
    const uint32_t inv = reciprocal_u32(heads);
    for (uint32_t x = 0; x < rows; ++x) {
        lanes::block_index = dim3(x);
        lanes::run_block(kBlock, [&] { join_pages_kernel<typename F::T, kPagedRows, true>(g, lanes_log2, rows, inv); });
    }
    for (uint32_t x = 0; x < ((rows << lanes_log2) + kBlock - 1) / kBlock; ++x) {
        lanes::block_index = dim3(x);
        lanes::run_block(kBlock, [&] { join_pages_kernel<typename F::T, kPagedRows, false>(g, lanes_log2, rows, inv); });
    }
}
void start_attend_pages_f32(const PagesArgs& g, const PagesForm&, hipStream_t) { run<PagedRows<In_f32, 64, false>>(g); }
void start_attend_pages_bf16(const PagesArgs& g, const PagesForm&, hipStream_t) { run<PagedRows<In_bf16, 64, false>>(g); }
void start_attend_pages_f16(const PagesArgs&, const PagesForm&, hipStream_t) { std::abort(); }

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

// An array with nothing behind it but what the sanitizer watches.
template <typename T>
static T* exactly(size_t n, int byte = 0) {
    void* p = nullptr;
    if (posix_memalign(&p, 64, n * sizeof(T) ? n * sizeof(T) : 1)) std::abort();
    std::memset(p, byte, n * sizeof(T));
    return static_cast<T*>(p);
}

struct Call {
    tom_oqm_pages_t g{};
    tom_oqm_view_t q{}, out{}, lse{};
    int32_t *table, *rows, *starts;
    int64_t* mask;
    int tokens = 0, heads, repeat, width = 1, n_pages = 2;
    std::vector<int32_t> good_rows, good_starts;
    Call(int heads_, int repeat_, int dtype, const std::vector<int>& had, const std::vector<int>& news, bool one_each) : heads(heads_), repeat(repeat_) {
        const int B = (int)had.size(), P = 16, D = 64, e = dtype == TOM_F32 ? 4 : 2;
        good_starts.push_back(0);
        for (int s = 0; s < B; ++s) {
            const int used = (had[s] + news[s] + P - 1) / P;
            n_pages += used;
            width = std::max(width, used + 1);
            good_rows.push_back(had[s]);
            good_starts.push_back(tokens += news[s]);
        }
        table = exactly<int32_t>((size_t)B * width);
        rows = exactly<int32_t>(B);
        starts = exactly<int32_t>(B + 1);
        for (int s = 0, at = 0; s < B; ++s)
            for (int i = 0; i < width; ++i) table[s * width + i] = i < (had[s] + news[s] + P - 1) / P ? at++ : -1;
        const size_t pool = (size_t)n_pages * heads * P * D;
        g.k = exactly<char>(pool * e);
        g.v = exactly<char>(pool * e);
        g.row_stride = D;
        g.head_stride = P * D;
        g.page_stride = (int64_t)heads * P * D;
        g.layer_stride = (int64_t)pool;
        g.n_layers = 1;
        g.n_pages = n_pages;
        g.heads = heads;
        g.page_rows = P;
        g.channels = D;
        g.dtype = dtype;
        g.table = table;
        g.rows = rows;
        g.starts = one_each ? nullptr : starts;
        g.sequences = B;
        g.table_pages = width;
        const size_t line = (size_t)heads * repeat * tokens;
        q.data = exactly<char>(line * D * e);
        q.heads = heads * repeat;
        q.rows = tokens;
        q.channels = D;
        q.dtype = dtype;
        q.row_stride = D;
        q.head_stride = (int64_t)tokens * D;
        out = q;
        out.data = exactly<char>(line * D * e);
        lse.data = exactly<float>(line);
        lse.heads = heads * repeat;
        lse.rows = tokens;
        lse.channels = 1;
        lse.dtype = TOM_F32;
        lse.row_stride = 1;
        lse.head_stride = tokens;
        mask = exactly<int64_t>(tokens, 0x55);
        good();
    }
    void good() {
        std::copy(good_rows.begin(), good_rows.end(), rows);
        std::copy(good_starts.begin(), good_starts.end(), starts);
    }
    void run(bool with_mask, int32_t left) {
        const size_t n = tom_oqm_attend_pages_workspace_bytes(&g, tokens, heads * repeat);
        int32_t* const ws = exactly<int32_t>((n + 3) / 4);
        for (size_t i = 0; i < n / 4; ++i) ws[i] = left;
        CHECK(tom_oqm_attend_pages(&g, 0, &q, &out, with_mask ? mask : nullptr, with_mask, 1, 0.125f, 0.0f, nullptr, nullptr, &lse, ws, n, nullptr) == TOM_OK);
        std::free(ws);
    }
};

// Starts, row counts and table entries of any kind, over what an earlier call may have left in the workspace.
static void numbers_that_make_no_sense() {
    std::mt19937 rng(3);
    auto some = [&](int B, int most, int least) {
        std::vector<int> v(B);
        for (int& x : v) x = least + (int)(rng() % (uint32_t)(most - least + 1));
        return v;
    };
    struct Kind {
        int heads, repeat, dtype, sequences, rows, tokens;
        bool one_each;
    };
    // parts of one sequence, of up to 64, of more; the same without parts; beyond those that are looked through; by position
    const Kind kinds[] = {{1, 3, TOM_BF16, 1, 700, 5, false}, {2, 5, TOM_BF16, 3, 300, 2, false}, {1, 2, TOM_BF16, 90, 300, 2, false}, {1, 1, TOM_F32, 70, 300, 3, false},
                          {2, 2, TOM_BF16, 60, 100, 2, false}, {2, 1, TOM_BF16, 80, 100, 3, false}, {1, 1, TOM_BF16, 600, 60, 1, false}, {1, 2, TOM_BF16, 20, 300, 1, true}};
    for (const Kind& k : kinds) {
        const int B = k.sequences;
        Call c(k.heads, k.repeat, k.dtype, some(B, k.rows, 0), some(B, k.tokens, k.one_each || B == 1 ? k.tokens : 0), k.one_each);
        const int T = c.tokens;
        const std::vector<int32_t> table(c.table, c.table + (size_t)B * c.width);
        for (int wrong = 0; wrong < 10; ++wrong) {
            c.good();
            std::copy(table.begin(), table.end(), c.table);
            for (int s = 0; s <= B; ++s) {
                if (wrong == 1) c.starts[s] = s ? 9999999 : 0;
                if (wrong == 2 || wrong == 9) c.starts[s] = s % 2 ? T : 0;
                if (wrong == 3) c.starts[s] = s % 2 ? 0 : T;
                if (wrong == 4) c.starts[s] = s ? T - s + 1 : -5;
                if (wrong == 5) c.starts[s] = (int32_t)rng();
                if (wrong == 6 || wrong == 7) c.starts[s] = (int32_t)(rng() % (uint32_t)(T + 1));
            }
            const int32_t ends[] = {-7, INT32_MAX, 0, INT32_MIN, c.width * 16};
            for (int s = 0; s < B && (wrong == 8 || wrong == 9); ++s) c.rows[s] = ends[(s + wrong) % 5];
            const int32_t entries[] = {INT32_MIN, INT32_MAX, c.n_pages, -1};
            for (size_t i = 0; i < table.size() && wrong == 9; i += 2) c.table[i] = entries[i / 2 % 4];
            for (int32_t left : {-1, 3}) {
                most_extra = 40;
                c.run(wrong % 2 != 0, left);
            }
        }
    }
    CHECK(blocks_run > 10000);
}

// The joins over sums of every kind, with a prior and without: without one nothing of it is looked at, whatever the sums are.
static void sums_that_are_none() {
    const float odd[] = {0.0f, 1.0f, 1e-45f, 1e-38f, 3e38f, INFINITY, -INFINITY, NAN};
    for (int dtype : {(int)TOM_BF16, (int)TOM_F32}) {
        Call c(1, 3, dtype, {900}, {5}, false);
        const size_t n = tom_oqm_attend_pages_workspace_bytes(&c.g, c.tokens, 3);
        CHECK(n > 0);
        for (float from : odd)
            for (float total : odd) {
                float* const ws = exactly<float>(n / 4);
                PagesArgs g{};
                CHECK(check_pages(&c.g, g.p) == TOM_OK);
                g.p.tokens = c.tokens;
                g.out = static_cast<char*>(c.out.data);
                g.out_row = 64 * (dtype == TOM_F32 ? 4 : 2);
                g.out_head = g.out_row * c.tokens;
                g.lse = static_cast<float*>(c.lse.data);
                g.lse_row = 1;
                g.lse_head = c.tokens;
                g.channels = 64;
                g.kv_heads = 1;
                g.repeat = 3;
                g.inv_repeat = reciprocal_u32(3);
                g.inv_kv_heads = reciprocal_u32(1);
                g.extra = g.items = 3;
                g.part_out = ws;
                g.part_stat = reinterpret_cast<f32pair*>(ws + 3 * 16 * 64);
                g.unit_first = reinterpret_cast<uint32_t*>(ws + 3 * 16 * 64 + 3 * 16 * 2);
                for (int i = 0; i < 3 * 16; ++i) g.part_stat[i] = f32pair{from, total};
                g.unit_first[0] = 0;
                g.unit_first[1] = 3;
                for (uint32_t x = 0; x < 15; ++x) {
                    lanes::block_index = dim3(x);
                    if (dtype == TOM_F32) lanes::run_block(kBlock, [&] { join_pages_kernel<In_f32, 16, true>(g, 4, 15, reciprocal_u32(3)); });
                    else lanes::run_block(kBlock, [&] { join_pages_kernel<In_bf16, 16, true>(g, 4, 15, reciprocal_u32(3)); });
                }
                lanes::block_index = dim3(0);
                if (dtype == TOM_F32) lanes::run_block(kBlock, [&] { join_pages_kernel<In_f32, 16, false>(g, 4, 15, reciprocal_u32(3)); });
                else lanes::run_block(kBlock, [&] { join_pages_kernel<In_bf16, 16, false>(g, 4, 15, reciprocal_u32(3)); });
                std::free(ws);
            }
    }
}

// What every workgroup finds, for each size of a block: inside the call whatever stands in starts and rows, and where those make sense each part of each block once.
template <int QT, int KT, int THREADS>
static void blocks(int heads, int repeat, const std::vector<int>& had, const std::vector<int>& news, int causal, bool parts) {
    std::mt19937 rng(5);
    Call c(heads, repeat, TOM_BF16, had, news, false);
    const int B = (int)had.size(), T = c.tokens;
    PagesArgs g{};
    CHECK(check_pages(&c.g, g.p) == TOM_OK);
    g.p.tokens = T;
    g.causal = causal;
    g.kv_heads = heads;
    g.repeat = repeat;
    g.inv_repeat = reciprocal_u32((uint32_t)repeat);
    g.least = 64;
    const uint32_t units = (uint32_t)pages_units(c.g, T, heads * repeat, QT);
    g.extra = parts ? 30 : 0;
    g.items = units + g.extra;
    g.sorted = !parts && B <= kMostSorted;
    for (int wrong = 0; wrong < (B > 100 ? 4 : 7); ++wrong) {
        c.good();
        for (int s = 0; s <= B; ++s) {
            if (wrong == 1) c.starts[s] = s % 2 ? T : 0;
            if (wrong == 2) c.starts[s] = s % 2 ? 0 : T;
            if (wrong == 3) c.starts[s] = s ? T - s + 1 : -5;
            if (wrong == 4) c.starts[s] = (int32_t)rng();
            if (wrong >= 5) c.starts[s] = (int32_t)(rng() % (uint32_t)(T + 1));
        }
        for (int s = 0; s < B && wrong >= 3; ++s) c.rows[s] = s % 3 ? (int32_t)rng() : INT32_MAX;
        std::vector<int> found_units(units, -1);
        long rows_seen = 0, rows_there = 0;
        for (uint32_t x = 0; x < g.items; ++x, ++blocks_run) {
            Block b{}, last_lanes{};
            bool there = false, last_there = false;
            static FoundItem shared;
            lanes::run_block(THREADS, [&] {
                Block mine{};
                const bool any = block_of<QT, KT, THREADS>(g, x, shared, mine);
                if (threadIdx.x == 0) there = any, b = mine;
                if (threadIdx.x == THREADS - 1) last_there = any, last_lanes = mine;
            });
            CHECK(there == last_there);
            if (!there) continue;
            CHECK(std::memcmp(&b, &last_lanes, sizeof b) == 0);
            const int32_t capacity = g.p.capacity;
            CHECK(b.sequence >= 0 && b.sequence < B);
            CHECK(b.tokens >= 1 && b.first_token >= 0 && (int64_t)b.first_token + b.tokens <= T);
            CHECK(b.tile >= 0 && (int64_t)b.tile * QT < (int64_t)b.tokens * repeat);
            CHECK(b.rows >= 0 && b.rows <= capacity && b.begin >= 0 && b.end <= capacity && b.for_all <= capacity);
            CHECK(parts ? b.first_item <= x && x < b.first_item + b.parts : b.parts == 1);
            const uint32_t unit = unit_of<QT>(g, b.sequence, b.first_token, b.tile);
            CHECK(unit < units);
            if (wrong == 0 && unit < units) {
                if (!parts || x == b.first_item) {
                    CHECK(found_units[unit] < 0);
                    found_units[unit] = b.sequence;
                }
                rows_seen += std::max(b.end - b.begin, 0);
            }
        }
        if (wrong > 0) continue;
        long blocks_found = 0, blocks_there = 0;
        for (int s : found_units) blocks_found += s >= 0;
        for (int s = 0; s < B; ++s) {
            const int tiles = (news[s] * repeat + QT - 1) / QT;
            blocks_there += tiles;
            for (int t = 0; t < tiles; ++t) {
                const int last = std::min((t + 1) * QT, news[s] * repeat) - 1;
                rows_there += std::min(had[s] + (causal ? last / repeat + 1 : news[s]), g.p.capacity);
            }
        }
        CHECK(blocks_found == blocks_there && rows_seen == rows_there);
    }
}
static void every_block_is_found() {
    std::mt19937 rng(9);
    for (int B : {1, 5, 64, 65, 300, 520})
        for (int causal : {0, 1})
            for (bool parts : {false, true}) {
                std::vector<int> had(B), news(B);
                const int most = B == 1 ? 300 : B < 64 ? 90 : B < 100 ? 14 : 4;
                for (int s = 0; s < B; ++s) {
                    had[s] = (int)(rng() % 300);
                    news[s] = B == 1 ? most : (int)(rng() % (uint32_t)most);
                }
                blocks<16, 32, 256>(1, 3, had, news, causal, parts);
                if (B < 100 || !causal) blocks<64, 32, 128>(1, 7, had, news, causal, parts);
                if (B < 100 || causal) blocks<128, 64, 256>(2, 5, had, news, causal, parts);
                if (B < 500 && !causal) blocks<256, 64, 512>(1, 9, had, news, causal, parts);
            }
}

int main() {
    sums_that_are_none();
    every_block_is_found();
    numbers_that_make_no_sense();
    if (failures) return 1;
    std::printf("pages lanes driver: clean, %d workgroups\n", blocks_run);
    return 0;
}
