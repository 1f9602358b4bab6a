// How the attention over chosen pages is cut, and how many pages entries span: every entry of a list in one part, lists that fit LDS, parts
// that a launch can hold.
#include <cstdio>
#include <initializer_list>

#include "../../paper_2411_10803_amd/csrc/cache4_plan.hpp"

static int g_bad = 0;
#define CHECK(c, ...) do { if (!(c) && g_bad++ < 20) { std::printf("line %d: ", __LINE__); std::printf(__VA_ARGS__); std::printf("\n"); } } while (0)

int main() {
    using namespace md;
    const int Bs[] = {1, 2, 7, 64, 1000}, Ns[] = {1, 2, 3, 5, 17, 160, 4000}, Gs[] = {1, 2, 3, 4, 5, 6, 8, 13, 16, 17, 40}, Hs[] = {1, 4, 32};
    const int budgets[] = {1, 2, 7, 16, 63, 64, 300, 1023, 1024, 1025, 5000, 1 << 20}, pages[] = {16, 64, 256}, tables[] = {0, 1, 90, 1024, 1025, 4096, 4097, 1 << 20};
    long together = 0, split = 0, eight = 0;
    for (int B : Bs) for (int N : Ns) for (int G : Gs) for (int H : Hs) for (int budget : budgets) for (int page : pages) for (int table : tables)
        for (int kind = 0; kind < 4; ++kind) {
            const bool f32 = kind & 1;
            const int d = kind & 2 ? 128 : 64;
            const C4Chosen c = c4_chosen(f32, d, B, N, G, H, budget, page, table);
            CHECK(c.tokens >= 1 && c.splits >= 1 && c.most >= 1 && c.most <= kC4ListMost, "B %d N %d G %d budget %d table %d", B, N, G, budget, table);
            CHECK(c.waves == 4 || (c.waves == 8 && !(f32 && d == 128) && c.splits == 1), "waves %d", c.waves);
            if (c.tokens > 1) {
                CHECK(c.tokens * G <= 16 && c.tokens <= N && c.splits == 1 && table > 0 && table <= kC4TableMost, "together: %d of %d", c.tokens, G);
                CHECK(c.most == table || c.most == c.tokens * budget, "together: a list of %d", c.most);
                // what lists are shared in lies where the rings will be: 2 bytes for each entry of the table
                CHECK(2 * (table + 1) <= c.waves * 2 * (32 * d + 256), "table %d", table);
                ++together;
            } else {
                CHECK((int64_t)c.splits * c.most >= budget && (int64_t)(c.splits - 1) * c.most < budget, "%d parts of %d for %d", c.splits, c.most, budget);
                const int64_t units = (int64_t)B * N * H * ((G + 15) / 16);
                CHECK(c.splits <= (budget + kC4ListMost - 1) / kC4ListMost || units * c.splits <= 512, "%d parts of %lld lists", c.splits, (long long)units);
            }
            const C4Chosen apart = c4_chosen(f32, d, B, N, G, H, budget, page, 0);       // what a workspace's size goes by
            CHECK(c.tokens > 1 || (c.splits == apart.splits && c.most == apart.most), "parts %d and %d", c.splits, apart.splits);
            split += c.splits > 1;
            eight += c.waves == 8;
        }
    CHECK(together > 0 && split > 0 && eight > 0, "a form that no call takes");
    CHECK(c4_choose_together(1, 256, 1000) && !c4_choose_together(1, 272, 1000) && c4_choose_together(136, 272, 1000), "few blocks");
    CHECK(!c4_choose_together(1 << 20, 2064, 1000) && !c4_choose_together(1 << 20, 256, 61441), "more than a block holds");
    for (int page : {16, 32, 256})
        for (int N = 1; N < 700; ++N) {
            int most = 0;
            for (int first = 0; first < page; ++first) {
                const int n = (first + N - 1) / page - first / page + 1;
                if (n > most) most = n;
            }
            CHECK(c4_span(N, page, 1 << 20) == most, "%d entries in pages of %d", N, page);
            CHECK(c4_span(N, page, 3) <= 3, "%d entries", N);
        }
    CHECK(c4_span(0x7FFFFFFF, 16, 1 << 26) == 1 << 26, "the longest");
    if (g_bad) { std::printf("%d wrong\n", g_bad); return 1; }
    std::printf("ok\n");
    return 0;
}
