// How csrc/cache4_plan.hpp cuts calls of the attention over the cache held in 4 bits: reads calls "f32 B N G H d capacity", one to a line, and
// prints "tile_rows tiles waves runs" for each.
#include <stdio.h>

#include "../../paper_2411_10803_amd/csrc/cache4_plan.hpp"

int main() {
    int f32, B, N, G, H, d;
    long capacity;
    while (scanf("%d %d %d %d %d %d %ld", &f32, &B, &N, &G, &H, &d, &capacity) == 7) {
        const md::C4Attend a = md::c4_attend(f32 != 0, B, N, G, H, d, capacity);
        printf("%d %d %d %d\n", a.tile_rows, a.tiles, a.waves, a.runs ? 1 : 0);
    }
    return 0;
}
