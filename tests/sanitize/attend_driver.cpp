// The arithmetic of the attention's rules at the ends of their ranges: built for the host with -fsanitize=address,undefined by
// tests/test_sanitizers_attend.py.  Exit status 0 = clean.
#include <cstdint>
#include <cstdio>

#include "oqm_attend.h"

static int failures = 0;
#define EXPECT(have, want)                                                                                        \
    do {                                                                                                          \
        const long long have_ = (long long)(have), want_ = (long long)(want);                                     \
        if (have_ != want_) {                                                                                     \
            std::fprintf(stderr, "line %d: %s = %lld, wanted %lld\n", __LINE__, #have, have_, want_);             \
            ++failures;                                                                                           \
        }                                                                                                         \
    } while (0)

// The causal edge: the last token sees every recent row, each one before it one less, also where rows or tokens are as many as a call takes.
static void causal_edge() {
    const int32_t rows[] = {0, 1, 2, 31, 4096, 1 << 20, 0x7fffffff - 4096}, tokens[] = {1, 2, 33, 4097, 1 << 20};
    for (int32_t r : rows)
        for (int32_t t : tokens)
            for (int32_t token : {0, t / 2, t - 1}) EXPECT(oqm::recent_seen(token, r, t), (int64_t)token + 1 + r - t);
}

int main() {
    causal_edge();
    if (failures) return 1;
    std::printf("attend driver: clean\n");
    return 0;
}
