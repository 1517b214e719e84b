// The rules of the attention over pages that go by numbers alone, at the ends of their ranges: built for the host with -fsanitize=address,undefined by
// tests/test_pages_rules.py.  Exit status 0 = clean.
#include <cstdint>
#include <cstdio>

#include "oqm_attend_pages.h"

using namespace oqm;

static int failures = 0;
#define CHECK(x)                                                          \
    do {                                                                  \
        if (!(x)) {                                                       \
            std::fprintf(stderr, "line %d: %s is false\n", __LINE__, #x); \
            ++failures;                                                   \
        }                                                                 \
    } while (0)

static tom_oqm_pages_t some_pages(int32_t heads, int32_t channels, int32_t dtype, int32_t sequences) {
    tom_oqm_pages_t g{};
    g.n_layers = g.n_pages = 1;
    g.heads = heads;
    g.page_rows = 64;
    g.channels = channels;
    g.dtype = dtype;
    g.starts = reinterpret_cast<const int32_t*>(uintptr_t{0x400000});
    g.sequences = sequences;
    g.table_pages = 100;
    return g;
}

// The form goes by the query rows of a KV head that a sequence has on average: up to 16, up to 64, up to 1024, more.
static void forms_go_by_the_average() {
    for (int32_t dtype : {(int32_t)TOM_BF16, (int32_t)TOM_F16, (int32_t)TOM_F32})
        for (int32_t sequences : {1, 2, 3, 48, 1000, 1 << 20})
            for (int32_t repeat : {1, 2, 7, 9, 15, 16, 17, 40, 64, 1000})
                for (int64_t most : {16, 64, 1024}) {
                    const int64_t last = most * sequences / repeat;  // tokens whose average is `most` or less
                    for (int64_t tokens = last - 1; tokens <= last + 2; ++tokens) {
                        if (tokens < 1 || tokens > 1 << 20 || tokens * repeat >= 1 << 30) continue;
                        const int32_t rows = pages_form(some_pages(1, 128, dtype, sequences), (int32_t)tokens, repeat).block_rows;
                        const bool within = tokens * repeat <= most * sequences;
                        if (dtype == TOM_F32) CHECK(rows == 16);
                        else if (most == 16) CHECK((rows == 16) == within);
                        else if (most == 64) CHECK((rows <= 64) == within);
                        else CHECK((rows <= 128) == within);
                    }
                }
}

int main() {
    forms_go_by_the_average();
    if (failures) return 1;
    std::printf("pages rules driver: clean\n");
    return 0;
}
