// CPU check of csrc/cache4_plan.hpp: the four regions of a page hold every byte once; entries of a block table and slots that name
// no page are told apart; a call's changes stay within the table's capacity; what one call takes, another puts back; and the scale
// byte is the smallest under which the largest magnitude rounds to 6 at most.
#include <stdio.h>
#include <math.h>
#include <string.h>
#include <random>
#include <vector>

#include "../../paper_2411_10803_amd/csrc/cache4_plan.hpp"

using namespace md;

static int g_bad = 0;
#define CHECK(c, ...) do { if (!(c)) { if (++g_bad <= 10) { printf("%s: ", #c); printf(__VA_ARGS__); printf("\n"); } } } while (0)

static void regions() {
    for (int d : {64, 128})
        for (int page : {16, 32, 64, 128, 256}) {
            std::vector<int> used(c4_page_bytes(page, d), 0);
            for (int t = 0; t < page; ++t) {
                for (int x = 0; x < d / 2; ++x) ++used.at(c4_k_codes(t, d) + x);
                for (int g = 0; g < d / 32; ++g) { ++used.at(c4_k_scales(page, t, d) + g); ++used.at(c4_v_scales(page, t, g, d)); }
                for (int part = 0; part < 16; ++part)
                    for (int x = 0; x < d / 32; ++x) ++used.at(c4_v_codes(page, t, part, d) + x);
            }
            for (size_t i = 0; i < used.size(); ++i) CHECK(used[i] == 1, "d=%d page=%d byte %zu used %d times", d, page, i, used[i]);
            // the attention's loads: sixteen tokens' K and four tokens' V of a lane, aligned to their width and within the page
            const int width = d / 8;
            for (int t0 = 0; t0 < page; t0 += 16)
                for (int lane = 0; lane < 64; ++lane) {
                    const int n = lane & 15, b = lane >> 4;
                    const int k = c4_k_codes(t0 + n, d) + b * width, v = c4_v_codes(page, t0 + 4 * b, n, d), s = c4_v_scales(page, t0 + 4 * b, n * d / 512, d);
                    CHECK(k % width == 0 && v % width == 0 && s % 4 == 0, "d=%d page=%d lane %d", d, page, lane);
                    CHECK(k + width <= (int)used.size() && v + width <= (int)used.size() && s + 4 <= (int)used.size(), "lane %d", lane);
                }
            CHECK(c4_page_bytes(page, d) % 16 == 0, "d=%d page=%d", d, page);
        }
}

static void names() {
    for (int n : {1, 5, 1000, 1 << 27}) {
        for (int id : {-2147483647 - 1, -1, n, 2147483647}) CHECK(c4_page_id(id, n) == -1, "%d of %d", id, n);
        for (int id : {0, n - 1}) CHECK(c4_page_id(id, n) == id, "%d of %d", id, n);
    }
    for (int shift : {4, 5, 8}) {
        const int n = 1000;
        for (int slot : {-2147483647 - 1, -1, n << shift, 2147483647}) CHECK(c4_slot(slot, n, shift).page == -1, "slot %d", slot);
        for (int slot : {0, 1, (n << shift) - 1}) {
            const C4Slot s = c4_slot(slot, n, shift);
            CHECK(s.page == slot >> shift && s.place == slot - (s.page << shift), "slot %d", slot);
        }
    }
}

static void changes() {
    for (int shift : {4, 6, 8})
        for (int entries : {1, 7, (1 << 30) >> 8})
            for (int len : {-2147483647 - 1, -5, 0, 1, 15, 16, 17, 100, 2147483647})
                for (int want : {-2147483647 - 1, -1, 0, 1, 16, 255, 256, 257, 2147483647}) {
                    const C4Change c = c4_change(len, want, entries, shift);
                    const int cap = entries << shift;
                    CHECK(c.old_len >= 0 && c.old_len <= cap && c.new_len >= 0 && c.new_len <= cap, "%d -> %d", len, want);
                    CHECK(c.held <= entries && c.need <= entries, "%d -> %d of %d", len, want, entries);
                    CHECK(c.need * (1l << shift) >= c.new_len && ((c.need - 1l) * (1l << shift) < c.new_len || c.new_len == 0), "%d pages of %d", c.need, c.new_len);
                }
}

// Random calls on a pool: every page is on the stack or in one request, and a call taken back leaves the stack as it was.
static void stack() {
    std::mt19937 rng(1);
    for (int round = 0; round < 300; ++round) {
        const int B = 1 + rng() % 9, entries = 1 + rng() % 12, shift = 4, pool = B * entries;
        std::vector<int> len(B, 0), free_pages(pool);
        std::vector<std::vector<int>> table(B, std::vector<int>(entries, -1));
        for (int i = 0; i < pool; ++i) free_pages[i] = i;
        int top = pool;
        auto call = [&](const std::vector<int>& want) {
            std::vector<int> gone;
            int taken = 0;
            for (int b = 0; b < B; ++b) {
                const C4Change c = c4_change(len[b], want[b], entries, shift);
                for (int e = c.need; e < c.held; ++e) gone.push_back(table[b][e]);
            }
            const int R = (int)gone.size();
            for (int j = 0; j < R; ++j) free_pages.at(c4_released_at(top, R, j)) = gone[j];
            for (int b = 0; b < B; ++b) {
                const C4Change c = c4_change(len[b], want[b], entries, shift);
                for (int e = c.held; e < c.need; ++e) table[b][e] = free_pages.at(c4_taken_at(top, R, taken++));
                len[b] = c.new_len;
            }
            top += R - taken;
        };
        std::vector<int> before = len, want(B);
        for (int step = 0; step < 6; ++step) {
            for (int& w : want) w = (int)(rng() % (entries * 16 + 1));
            call(want);
            std::vector<int> seen(pool, 0);
            for (int i = 0; i < top; ++i) ++seen[free_pages[i]];
            for (int b = 0; b < B; ++b)
                for (int e = 0; e < c4_pages_of(len[b], shift); ++e) ++seen[table[b][e]];
            for (int i = 0; i < pool; ++i) CHECK(seen[i] == 1, "page %d %d times", i, seen[i]);
        }
        // grow and shrink back
        const std::vector<int> old_len = len, old_free(free_pages.begin(), free_pages.begin() + top);
        for (int b = 0; b < B; ++b) want[b] = len[b] + (int)(rng() % (entries * 16 + 1 - len[b]));
        call(want);
        call(old_len);
        CHECK(top == (int)old_free.size(), "height %d", top);
        for (int i = 0; i < top; ++i) CHECK(free_pages[i] == old_free[i], "place %d", i);
    }
}

static void scales() {
    std::mt19937 rng(2);
    for (long n = 0; n < 2000000; ++n) {
        uint32_t bits = rng() & 0x7FFFFFFFu;
        if (n < 40000) bits = (uint32_t)(n / 160) << 23 | (n % 160 < 80 ? (uint32_t)(n % 80) : 0x600000u + (uint32_t)(n % 80) - 40u);
        float a;
        memcpy(&a, &bits, 4);
        const int code = c4_scale_code(bits);
        if (!std::isfinite(a)) { CHECK(code == 255, "%08x", bits); continue; }
        int want = 27;
        while (want < 252 && (double)a >= 7.0 * ldexp(1.0, want - 127)) ++want;
        CHECK(code == want, "%g: %d, not %d", a, code, want);
    }
}

int main() {
    regions();
    names();
    changes();
    stack();
    scales();
    printf("%d bad\n", g_bad);
    return g_bad != 0;
}
