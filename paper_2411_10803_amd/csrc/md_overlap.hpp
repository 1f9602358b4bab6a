// Do two ranges of bytes, or two tensors of rows, share one?  Without any HIP header, for the CPU tests.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace md {

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + nb && pb < pa + na;
}

// Runs of `run` bytes on a grid of up to three axes: strides in bytes, the largest first, each at least as long as what lies within it;
// axes with one place are left out.
struct ByteGrid {
    const void* p;
    int axes;
    int64_t stride[3], n[3], run;
    // Bytes from the first to the last one, of what lies within axis `from` - 1.
    int64_t extent(int from) const {
        int64_t e = run;
        for (int x = from; x < axes; ++x) e += (n[x] - 1) * stride[x];
        return e;
    }
};
inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }       // b > 0
// `delta`: from a's first byte to b's, of what lies within their outer x axes.  Where the next axes have one stride, as those of views of one
// tensor, places of the two are looked at whose extents meet: two at most, as neither is longer than the stride.  Where they have not, extents
// that meet are taken as sharing a byte.
inline bool grids_meet(int64_t delta, const ByteGrid& a, const ByteGrid& b, int x) {
    if (delta >= a.extent(x) || -delta >= b.extent(x)) return false;
    if (x >= a.axes && x >= b.axes) return true;
    if (x >= a.axes || x >= b.axes || a.stride[x] != b.stride[x]) return true;
    const int64_t s = a.stride[x], ea = a.extent(x + 1), eb = b.extent(x + 1);
    int64_t from = floor_div(-eb - delta, s) + 1, to = floor_div(ea - 1 - delta, s);     // -eb < delta + m s < ea
    if (from < 1 - a.n[x]) from = 1 - a.n[x];
    if (to > b.n[x] - 1) to = b.n[x] - 1;
    for (int64_t m = from; m <= to; ++m)
        if (grids_meet(delta + m * s, a, b, x + 1)) return true;
    return false;
}
inline bool overlaps(const ByteGrid& a, const ByteGrid& b) {
    if (!a.p || !b.p) return false;
    return grids_meet((int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)), a, b, 0);
}

}  // namespace md
