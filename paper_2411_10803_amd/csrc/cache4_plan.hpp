// The cache held in 4 bits: where things lie in a page, and the arithmetic of block tables and slots.  Plain arithmetic of the host
// and of the kernels, without any HIP header, so that a CPU test can compile it.
#pragma once
#include <stdint.h>

#ifndef MD_PLAN_FN
#ifdef __HIPCC__
#define MD_PLAN_FN __host__ __device__ __forceinline__
#else
#define MD_PLAN_FN inline
#endif
#endif

namespace md {
namespace {

// A page of `page` tokens of one head, byte offsets (16-byte aligned regions, as page is a multiple of 16):
//   K codes [page][d/2] | K scales [page][d/32] | V codes [page/4][16][4][d/32] | V scales [page/4][d/32][4]
// K is laid out for the product S = K Q^T, where a lane of a wave wants channels of one token; V for O = V^T P^T, where it
// wants tokens of one channel: four tokens' codes of the d/16 channels that a lane deals with are one load.
MD_PLAN_FN int c4_page_bytes(int page, int d) { return page * (d + d / 16); }
MD_PLAN_FN int c4_k_codes(int t, int d) { return t * (d / 2); }                                            // + channel / 2
MD_PLAN_FN int c4_k_scales(int page, int t, int d) { return page * (d / 2) + t * (d / 32); }               // + channel / 32
// + (channel % (d/16)) / 2, of the token's sixteenth `part` = channel / (d/16)
MD_PLAN_FN int c4_v_codes(int page, int t, int part, int d) { return page * (d / 2 + d / 32) + ((t / 4) * 16 + part) * (d / 8) + (t % 4) * (d / 32); }
MD_PLAN_FN int c4_v_scales(int page, int t, int group, int d) { return page * (d + d / 32) + (t / 4) * (d / 8) + group * 4 + t % 4; }

MD_PLAN_FN int c4_clamp(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }
// pages of n tokens
MD_PLAN_FN int c4_pages_of(int n, int page_shift) { return (int)(((uint32_t)n + (1u << page_shift) - 1u) >> page_shift); }

// What a call of cache4_pages does for one request: its lengths within the table's capacity, and its pages before and after.
struct C4Change { int old_len, new_len, held, need; };
MD_PLAN_FN C4Change c4_change(int len, int new_len, int max_pages, int page_shift) {
    const int cap = max_pages << page_shift;                      // the host checks that this fits 31 bits
    C4Change c;
    c.old_len = c4_clamp(len, 0, cap);
    c.new_len = c4_clamp(new_len, 0, cap);
    c.held = c4_pages_of(c.old_len, page_shift);
    c.need = c4_pages_of(c.new_len, page_shift);
    return c;
}
// The stack of free pages, `top` entries high: the released pages go on it, the first of them uppermost, then the taken ones come
// off it, so that a call that undoes another leaves the stack as it was.  Places of the j-th released and the j-th taken page.
MD_PLAN_FN int c4_released_at(int top, int released, int j) { return top + released - 1 - j; }
MD_PLAN_FN int c4_taken_at(int top, int released, int j) { return top + released - 1 - j; }

// An entry of the block table, or -1 where it names no page of the pool.
MD_PLAN_FN int c4_page_id(int id, int n_pages) { return (uint32_t)id < (uint32_t)n_pages ? id : -1; }
// A slot's page and place; page -1 where the slot names none.
struct C4Slot { int page, place; };
MD_PLAN_FN C4Slot c4_slot(int slot, int n_pages, int page_shift) {
    if (slot < 0) return C4Slot{-1, 0};
    return C4Slot{c4_page_id(slot >> page_shift, n_pages), slot & ((1 << page_shift) - 1)};
}

// The byte of a group's scale from the bits of its largest magnitude (fp32, sign removed): the power of two under which the
// magnitude rounds to 6 at most.  Adding 1/4 to the mantissa carries into the exponent from 1.75 on.
MD_PLAN_FN int c4_scale_code(uint32_t most) {
    if (most >= 0x7F800000u) return 255;                          // an infinity or a NaN in the group
    return c4_clamp((int)((most + 0x200000u) >> 23) - 2, 27, 252);
}

// How the attention is cut over blocks of equal work.  A sample's work is H * tiles units (a K/V head and a tile of query rows) of
// `steps` 32-key steps each, in this order, one sample after the other; a block takes a run of consecutive steps.
struct C4Work { int tiles, steps; };
MD_PLAN_FN C4Work c4_work(int length, int rows, int tile_rows) {
    C4Work w;
    w.tiles = (rows + tile_rows - 1) / tile_rows;
    w.steps = length > 0 ? (length + 31) >> 5 : 1;                // (rows that see no key are written by somebody too)
    return w;
}
// Blocks that get a run: `least` steps each at least, where there are that many.
MD_PLAN_FN int c4_runs(int total, int blocks, int least) { return c4_clamp(total / least, 1, blocks); }
MD_PLAN_FN int c4_run_begin(int p, int total, int runs) { return (int)((int64_t)total * p / runs); }
// The run that holds step `at`.
MD_PLAN_FN int c4_run_of(int at, int total, int runs) { return (int)((((int64_t)at + 1) * runs - 1) / total); }
// Where run p leaves the sums of a unit that it holds only a part of, of its two places: the second one for the unit that its run ends
// in and begins with or before, the first one for the unit that began in an earlier run.
MD_PLAN_FN int c4_part_place(int p, int unit_begin, int total, int runs) { return 2 * p + (c4_run_begin(p, total, runs) > unit_begin ? 0 : 1); }

// How a call of the attention is cut up: by what the host knows, which is the tables' capacity and not the samples' lengths.
//   tile_rows  query rows of a unit.  Of the G query heads of a K/V head and the N tokens, sixteen fill a matrix tile.  Two tiles to a
//              unit convert each key once for 32 rows instead of 16, but leave half as many units and three blocks to a CU instead of four:
//              they pay from about three units per CU on, and from two to three it is one or the other.  us with 16 / 32 rows, by units of 16:
//              4 x 512 tokens of 32 heads on 8, up to 5888 keys (4096) 313 / 233, 16 x 128 of 32 heads, 704 keys (4096) 72 / 63, 8 x 512 of 32
//              heads, 512 keys (8192) 96 / 84, 1 x 512 of 32 heads on 8, 6000 keys (1024) 116 / 103; drafts of 4 tokens, 64 heads on 8, up to
//              2000 keys, 128 of them (2048) 75 / 55, 64 (1024) 40 / 36; of 5 tokens, 32 heads on 4, 64 of them (768) 37 / 35; 1 x 320 of 32
//              heads, 2000 keys (640) 36 / 38; 33 drafts of 4 tokens, 64 heads on 8 (528), up to 1000 keys 20.6 / 20.2, up to 4000 43 / 51;
//              1 x 128, 1000 keys (256) 13 / 17, 1 x 64 of 32 heads, 4000 keys (128) 26 / 35
//   runs       blocks of equal work, joined by a second kernel, instead of a block per unit.  Where there are few units, a block of
//              eight waves takes 4.5 us + 0.15 us per 32 keys, the runs take 12 us and more with their work, and have all CUs; where
//              sequences may be very long, one of them among short ones must not be left to one block.  Lengths are often well
//              below the tables' capacity, which is all that the host knows.  us, a block per unit / runs: 8 units of 3200 keys 19 / 12, of
//              16000 78 / 16, 32 of 640 7.4 / 10, of 2000 14.7 / 14.8, of 2560 16.7 / 12.9, of 4000 24 / 17, of 1000 in tables of 4096 9.6 /
//              10.5, 128 of 2560 18 / 23, of 4000 25 / 23, of up to 2000 in tables of 4096 15 / 20, 160 of 6000 40 / 38, of 9000 52 / 48, 256 of
//              2000 18 / 23, 512 of 4000 53 / 58; 16 units of up to 100000 keys 458 / 45
//   waves      of a block per unit: eight (four: 64 sequences of up to 4000 keys and 32 heads 122 us instead of 117, 32 units of 2000 keys
//              17.8 instead of 14.6); four where a wave takes more registers, where a unit has no more than eight steps, and where there
//              are more units than the 512 blocks of eight waves that run at a time and no long ones.  us with four / eight: units of up
//              to 1000 keys in tables of 2000, 640 of them 20.5 / 22.0, 1024 24 / 27.5, 2048 38 / 45.5, 512 16.6 / 16.9, 256 12.8 / 11.7; of up
//              to 300 in 600, 2048 22 / 30; of d = 64, 1000 in 2000, 2048 29 / 36; 1024 of up to 2000 in 4000 41 / 38
struct C4Attend { int tile_rows, tiles, waves; bool runs; };
constexpr int kC4Blocks = 1024;                      // of the runs: four to a CU
constexpr int kC4Least = 4;                          // steps of a run, one per wave of its block
inline C4Attend c4_attend(bool f32, int B, int N, int G, int H, int d, int64_t capacity) {
    const int64_t rows = (int64_t)N * G, steps = (capacity + 31) / 32;
    C4Attend a;
    a.tile_rows = !f32 && rows > 16 && (int64_t)B * H * ((rows + 15) / 16) > 512 ? 32 : 16;
    a.tiles = (int)((rows + a.tile_rows - 1) / a.tile_rows);
    const int64_t units = (int64_t)B * H * a.tiles;
    // (a run's steps are counted in 31 bits)
    a.runs = (steps * (200 - units) > 16000 || steps > 512) && units < 0x7FFFFFFFl / steps;
    a.waves = a.runs || a.tile_rows == 32 || (f32 && d == 128) || steps <= 8 || (steps <= 64 && units > 512) ? 4 : 8;
    return a;
}

// Pages that N consecutive entries may lie in.
inline int c4_span(int N, int page, int max_pages) {
    const int64_t most = ((int64_t)N + page - 2) / page + 1;
    return most < max_pages ? (int)most : max_pages;
}

// Whether a call of the choice scores and chooses in one launch: up to 2048 pages, whose scores a block has in LDS.  A block then reads all of
// its pages' bounds by itself, which takes long where there are few blocks.  us in two launches / in one, by blocks and pages: 8 of 119
// 8.3 / 5.5, of 244 8.2 / 7.7, of 494 8.3 / 11.4, of 994 8.3 / 18; 32 of 244 8.8 / 7.6; 128 of 244 8.6 / 7.6, of 494 10 / 11.7, of 1994 18 / 31;
// 256 of 994 18 / 20; 512 of 375 36 / 23, of 994 29 / 30, of 1994 66 / 65; 640 of 1875 56 / 63; 1024 of 1994 128 / 115; 1280 of 94 23 / 10, of
// 375 36 / 22, of 688 99 / 78, of 994 62 / 56; 2048 of 128 22 / 15
inline bool c4_choose_together(int64_t blocks, int pitch, size_t lds) {
    return pitch <= 2048 && lds <= 61440 && (pitch <= 256 || blocks * 2 >= pitch);
}

// A launch has fewer than 2^32 threads along x: lists of the choice with a block of `threads` threads each, in how many blocks along x, and along y.
struct C4Lists { int x, y; };
inline C4Lists c4_lists(int lists, int threads) {
    const int most = (int)(0x80000000u / (unsigned)threads);
    return lists <= most ? C4Lists{lists, 1} : C4Lists{most, (int)(((int64_t)lists + most - 1) / most)};
}

// How the attention over chosen pages is cut.
//   tokens   that a block takes together, as many as fill 16 query rows with their heads: over all of the pages that any of them has chosen.
//            What a key costs is then shared, but where tokens choose different pages there are more of them to go through and fewer blocks.
//            It pays where there are blocks for the chip without it.  us apart / together where tokens choose at random, and where they
//            choose the same, 1024 keys of about 6000: 1 x 64 tokens of 40 heads 55 / 27, 53 / 13; 4 x 128 of 32 heads on 8 83 / 70, 80 / 27; of
//            64 on 8, two together, 82 / 79, 81 / 49; 64 x 4 of 32 heads 180 / 130, 153 / 54; 4 x 16 of 32 heads, 512 keys 30 / 26, 29 / 12;
//            2 x 200 of 28 on 4 40 / 43, 38 / 26; but 1 x 16 of 32 on 8 12 / 25, 12 / 13; 16 x 5 of 32 on 8 22 / 28, 21 / 14; 64 x 2 of 32 on 8
//            31 / 32, 26 / 19
//   splits   parts of a token's list, a block each, joined by a second launch: where there are few lists and they are long, up to 512 blocks
//            of eight steps of 32 keys or more.  us in one part / in 4 / 8 / 16 / 32: 8 lists of 32 steps 11.6 / 12.0 / 11.7 / 11.4, of 64 15.9 /
//            13.7 / 12.3 / 11.4 / 11.5, of 128 25 / 17 / 14.0 / 12.8 / 11.8, of 256 44 / 23 / 17 / 14.2 / 12.7, of 1024 159 / 65 / 38 / 25 / 20; 32 of
//            32 11.1 / 12.5 / 11.9 / 12.8, of 64 16.1 / 14.6 / 12.8 / 13.9 / 13.5, of 128 25 / 18 / 15.1 / 15.6 / 16.3, of 512 83 / 38 / 25 / 23 / 24; 128 of
//            64 17.4 / 18.9 / 19.3, of 128 27 / 23 / 24, of 512 86 / 57 / 56; but 256 of 128 29 / 34 / 37
//   most     entries of a list to a part (tokens > 1: of the list of all)
//   waves    of a block: eight while there are no more than 512 blocks.  us with four / eight: 8 lists of 32 steps 12.5 / 13.0, of 64 18.9 / 16.5,
//            of 128 32 / 25; 512 of 32 17.8 / 17.4; 640 of 32 22.6 / 26; 5120 of 32 86 / 113
struct C4Chosen { int tokens, splits, most, waves; };
constexpr int kC4ListMost = 1024;                    // entries of a list in LDS
constexpr int kC4TableMost = 4096;                   // of a block table that lists are shared in: 2 bytes each lie in LDS
inline C4Chosen c4_chosen(bool f32, int d, int B, int N, int G, int H, int budget, int page, int max_pages) {
    C4Chosen c;
    const int64_t apart = (int64_t)B * N * H * ((G + 15) / 16), steps = ((int64_t)budget * page + 31) / 32;
    const int most_waves = f32 && d == 128 ? 4 : 8;
    c.tokens = G <= 8 && N > 1 && apart >= 1536 && max_pages > 0 && max_pages <= kC4TableMost ? (N < 16 / G ? N : 16 / G) : 1;
    const int64_t together = (int64_t)c.tokens * budget, most = together < max_pages ? together : max_pages;
    if (c.tokens > 1 && most <= kC4ListMost) {
        c.splits = 1;
        c.most = (int)most;
        c.waves = (int64_t)B * ((N + c.tokens - 1) / c.tokens) * H <= 512 ? most_waves : 4;
        return c;
    }
    c.tokens = 1;
    const int64_t parts = steps / 8 < 512 / apart ? steps / 8 : 512 / apart, need = (budget + kC4ListMost - 1) / kC4ListMost;
    c.splits = (int)(parts > 4 || (parts > 2 && steps > 64) ? (parts < budget ? parts : budget) : 1);
    if (c.splits < need) c.splits = (int)need;
    c.most = (budget + c.splits - 1) / c.splits;
    c.splits = (budget + c.most - 1) / c.most;
    c.waves = apart * c.splits <= 512 && c.splits == 1 ? most_waves : 4;
    return c;
}

}  // namespace
}  // namespace md
