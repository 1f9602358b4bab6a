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
            CHECK(c4_page_bytes(page, d) % 64 == 0, "d=%d page=%d", d, page);
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

// The attention's cut: what the tests of the GPU rely on, and limits.
static void forms() {
    auto is = [](const C4Attend& a, int tile_rows, int waves, bool runs) { return a.tile_rows == tile_rows && a.waves == waves && a.runs == runs; };
    CHECK(is(c4_attend(false, 3, 1, 1, 2, 128, 3040), 16, 4, true), "few units");
    CHECK(is(c4_attend(false, 16, 1, 1, 2, 128, 112), 16, 4, false), "short");
    CHECK(is(c4_attend(false, 16, 1, 1, 2, 128, 512), 16, 8, false), "eight waves");
    CHECK(is(c4_attend(true, 16, 1, 1, 2, 128, 512), 16, 4, false) && is(c4_attend(true, 16, 1, 1, 2, 64, 512), 16, 8, false), "fp32");
    CHECK(is(c4_attend(false, 22, 20, 1, 13, 64, 512), 32, 4, false), "two tiles");
    CHECK(is(c4_attend(true, 22, 20, 1, 13, 64, 512), 16, 4, false), "two tiles, fp32");
    CHECK(is(c4_attend(false, 22, 20, 1, 13, 128, 16640), 32, 4, true), "two tiles in runs");
    CHECK(is(c4_attend(false, 16, 1, 1, 16, 64, 16640), 16, 4, true), "very long");
    std::mt19937 rng(3);
    for (int n = 0; n < 200000; ++n) {
        const int B = 1 << (rng() % 16), N = 1 + rng() % (1 << (rng() % 12)), G = 1 + rng() % 16, H = 1 << (rng() % 7), d = rng() % 2 ? 64 : 128;
        const int64_t cap = 16 + rng() % (1 << (4 + rng() % 26));
        const C4Attend a = c4_attend(rng() % 4 == 0, B, N, G, H, d, cap);
        const int64_t units = (int64_t)B * H * a.tiles, steps = (cap + 31) / 32;
        CHECK((int64_t)a.tiles * a.tile_rows >= (int64_t)N * G && ((int64_t)a.tiles - 1) * a.tile_rows < (int64_t)N * G, "tiles");
        CHECK(!a.runs || units * steps < 0x7FFFFFFFl, "%d %d: steps", B, N);
        CHECK(a.waves == 4 || a.waves == 8, "waves");
    }
}

// Runs over samples of any length: every step of every unit is in one run, what a run leaves of a unit lies where the join looks for it, and
// nowhere else.
static void runs() {
    std::mt19937 rng(4);
    for (int round = 0; round < 3000; ++round) {
        const int B = 1 + rng() % 7, H = 1 + rng() % 4, rows_of = rng() % 3, blocks = 1 + rng() % 40, least = 1 + rng() % 5;
        std::vector<C4Work> work;
        std::vector<int> begin;
        int total = 0;
        for (int b = 0; b < B; ++b) {
            const int length = rng() % 4 ? (int)(rng() % (1 << (rng() % 11))) : 0, rows = rows_of == 0 ? 1 : (int)(rng() % 70);
            work.push_back(c4_work(length, rows, 16));
            begin.push_back(total);
            total += H * work[b].tiles * work[b].steps;
        }
        if (total == 0) continue;
        const int n = c4_runs(total, blocks, least);
        CHECK(n >= 1 && n <= blocks && (n == 1 || total / n >= least), "%d runs of %d", n, total);
        CHECK(c4_run_begin(0, total, n) == 0 && c4_run_begin(n, total, n) == total, "ends");
        std::vector<int> place(2 * blocks, -1);      // first step of the unit whose part lies there
        std::vector<char> done(total, 0);
        for (int p = 0; p < n; ++p) {
            int at = c4_run_begin(p, total, n), b = 0;
            const int stop = c4_run_begin(p + 1, total, n);
            while (at < stop) {
                while (at - begin[b] >= H * work[b].tiles * work[b].steps) ++b;
                const int unit = (at - begin[b]) / work[b].steps, first = at - begin[b] - unit * work[b].steps;
                const int last = first + stop - at < work[b].steps ? first + stop - at : work[b].steps, unit_begin = begin[b] + unit * work[b].steps;
                for (int i = first; i < last; ++i) { CHECK(!done[unit_begin + i], "step twice"); done[unit_begin + i] = 1; CHECK(c4_run_of(unit_begin + i, total, n) == p, "run of a step"); }
                if (first || last < work[b].steps) {
                    const int to = c4_part_place(p, unit_begin, total, n);
                    CHECK(to >= 0 && to < 2 * blocks && place[to] < 0, "place %d", to);
                    place[to] = unit_begin;
                }
                at += last - first;
            }
        }
        for (int i = 0; i < total; ++i) CHECK(done[i], "step %d of %d left out", i, total);
        int parts = 0, found = 0;
        for (int x : place) parts += x >= 0;
        for (int b = 0; b < B; ++b)
            for (int u = 0; u < H * work[b].tiles; ++u) {
                const int first = begin[b] + u * work[b].steps;
                const int p0 = c4_run_of(first, total, n), p1 = c4_run_of(first + work[b].steps - 1, total, n);
                if (p0 == p1) continue;
                for (int p = p0; p <= p1; ++p) { CHECK(place[c4_part_place(p, first, total, n)] == first, "part of run %d", p); ++found; }
            }
        CHECK(found == parts, "%d parts, %d looked for", parts, found);
    }
}

int main() {
    forms();
    runs();
    regions();
    names();
    changes();
    stack();
    scales();
    printf("%d bad\n", g_bad);
    return g_bad != 0;
}
