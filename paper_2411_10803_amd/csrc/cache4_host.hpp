// The cache held in 4 bits, on the host: what its calls check alike.
#pragma once
#include "cache4_device.hpp"

#include <cmath>

namespace md {
namespace {

// What all calls share: the pool's shape.
int check_pool(const char* who, int H, int d, int n_pages, int page, int max_pages, Pool* p) {
    if (H <= 0 || d <= 0 || n_pages <= 0 || page <= 0 || max_pages <= 0) return fail(MD_EINVAL, "%s: sizes must be positive", who);
    if (d != 64 && d != 128) return fail(MD_ESHAPE, "%s: d=%d is not supported (64 or 128)", who, d);
    if (page < 16 || page > 256 || (page & (page - 1))) return fail(MD_ESHAPE, "%s: page=%d must be a power of two from 16 to 256", who, page);
    if ((long)n_pages * page > 0x7FFFFFFFl) return fail(MD_ESHAPE, "%s: a pool of %d pages of %d tokens has more slots than 31 bits name", who, n_pages, page);
    if ((long)max_pages * page > 0x7FFFFFFFl / 2) return fail(MD_ESHAPE, "%s: %d pages of %d tokens are too many for one request", who, max_pages, page);
    if (H > 65535) return fail(MD_ESHAPE, "%s: H=%d out of range", who, H);
    if ((long)n_pages * H * c4_page_bytes(page, d) > (256l << 30)) return fail(MD_ESHAPE, "%s: a pool of more than 256 GiB", who);
    *p = Pool{n_pages, page, __builtin_ctz((unsigned)page), max_pages, H, (long)c4_page_bytes(page, d)};
    return MD_OK;
}
size_t pool_bytes(const Pool& p) { return (size_t)p.n_pages * p.H * p.stride; }

int check_dtype(const char* who, int dtype) {
    return dtype == MD_F32 || dtype == MD_BF16 ? MD_OK : fail(MD_EDTYPE, "%s: unknown dtype %d", who, dtype);
}

// A launch has fewer than 2^32 threads along x: of the copies 16 per row, of the attention up to 512 per tile of query rows.
constexpr long kMaxRows = (1l << 28) - 16, kMaxUnits = (1l << 23) - 1;

struct Range { const void* p; size_t n; };
// An output that shares no byte with any of some ranges.
int check_apart(const char* who, const Range& out, const Range* r, int all) {
    for (int c = 0; c < all; ++c)
        if (overlaps(out.p, out.n, r[c].p, r[c].n)) return fail(MD_EALIAS, "%s: the outputs, the workspace and the inputs must not overlap", who);
    return MD_OK;
}
// None of the first `outs` ranges may share a byte with any other range.
int check_apart(const char* who, const Range* r, int outs, int all) {
    int rc = MD_OK;
    for (int a = 0; a < outs && rc == MD_OK; ++a) rc = check_apart(who, r[a], r + a + 1, all - a - 1);
    return rc;
}

size_t rows_bytes(const KvLayout& l, int B, int N, int H, int d, int dtype) { return layout_extent_bytes(l, B, N, H, d) / 2 * elt_size(dtype); }
// The bytes of rows, without what lies between them: views of one projection's output share none, though their extents do.
ByteGrid rows_grid(const void* p, const KvLayout& l, int B, int N, int H, int d, int dtype) {
    const int64_t e = (int64_t)elt_size(dtype), stride[3] = {l.batch * e, l.token * e, l.head * e}, n[3] = {B, N, H};
    ByteGrid g{p, 0, {}, {}, d * e};
    for (int x = 0; x < 3; ++x) {
        if (n[x] < 2) continue;
        int at = g.axes++;
        for (; at > 0 && g.stride[at - 1] < stride[x]; --at) { g.stride[at] = g.stride[at - 1]; g.n[at] = g.n[at - 1]; }
        g.stride[at] = stride[x];
        g.n[at] = n[x];
    }
    return g;
}

}  // namespace
}  // namespace md
