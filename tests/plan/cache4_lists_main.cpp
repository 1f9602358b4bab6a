// Blocks of the choice, one to a list: a launch has fewer than 2^32 threads along x, and every list has a block.
#include <cstdio>
#include <initializer_list>

#include "../../paper_2411_10803_amd/csrc/cache4_plan.hpp"

int main() {
    int bad = 0;
    for (int threads : {256, 1024})
        for (int lists : {1, 2, 255, 65536, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, 5000000, 3 << 21, (1 << 23) - 2, (1 << 23) - 1}) {
            const md::C4Lists l = md::c4_lists(lists, threads);
            const long blocks = (long)l.x * l.y;
            if (l.x < 1 || l.y < 1 || l.y > 65535 || (unsigned long)l.x * threads >= 1ul << 32 || blocks < lists || blocks - l.x >= lists || blocks >= 1l << 31) {
                std::printf("%d lists of %d threads: %d x %d\n", lists, threads, l.x, l.y);
                ++bad;
            }
            if (l.y > 1 && (long)lists * threads < 1l << 31) ++bad;          // (one row of blocks wherever that fits)
        }
    std::printf(bad ? "%d wrong\n" : "ok\n", bad);
    return bad != 0;
}
