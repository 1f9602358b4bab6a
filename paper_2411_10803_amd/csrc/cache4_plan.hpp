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

}  // namespace
}  // namespace md
