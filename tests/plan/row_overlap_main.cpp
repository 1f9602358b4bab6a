// Whether two tensors of rows share a byte: against every byte of small grids.
#include <cstdio>
#include <cstdlib>
#include <set>

#include "../../paper_2411_10803_amd/csrc/md_overlap.hpp"

static unsigned g_state = 1;
static int below(int n) { g_state = g_state * 1664525u + 1013904223u; return (int)((g_state >> 8) % (unsigned)n); }

static md::ByteGrid grid(const char* p, int axes, const long* stride, const long* n, long run) {
    md::ByteGrid g{p, axes, {}, {}, run};
    for (int x = 0; x < axes; ++x) { g.stride[x] = stride[x]; g.n[x] = n[x]; }
    return g;
}
static std::set<const char*> bytes(const md::ByteGrid& g) {
    std::set<const char*> s;
    const long n0 = g.axes > 0 ? g.n[0] : 1, n1 = g.axes > 1 ? g.n[1] : 1, n2 = g.axes > 2 ? g.n[2] : 1;
    for (long a = 0; a < n0; ++a) for (long b = 0; b < n1; ++b) for (long c = 0; c < n2; ++c) for (long r = 0; r < g.run; ++r)
        s.insert(static_cast<const char*>(g.p) + a * (g.axes > 0 ? g.stride[0] : 0) + b * (g.axes > 1 ? g.stride[1] : 0) + c * (g.axes > 2 ? g.stride[2] : 0) + r);
    return s;
}
static bool share(const std::set<const char*>& a, const std::set<const char*>& b) {
    for (const char* x : a) if (b.count(x)) return true;
    return false;
}

int main() {
    static char memory[1 << 16];
    int bad = 0;
    long apart = 0, meet = 0, within = 0;
    for (int it = 0; it < 60000; ++it) {
        const int axes = below(4);
        const long run = 1 + below(4);
        long stride[3], na[3], nb[3], nc[3], room = run;
        for (int x = axes - 1; x >= 0; --x) {                                // the innermost axis first; grids of up to room / stride places
            stride[x] = room + below(6);
            const long most = 1 + below(3);
            na[x] = 1 + below((int)most);
            nb[x] = 1 + below((int)most);
            nc[x] = most;
            room = stride[x] * nc[x] + below(5);
        }
        const md::ByteGrid a = grid(memory + (1 << 15), axes, stride, na, run), b = grid(a.p ? memory + (1 << 15) + below((int)(2 * room + 8)) - room - 4 : 0, axes, stride, nb, 1 + below((int)run));
        const std::set<const char*> ba = bytes(a), bb = bytes(b);
        const bool want = share(ba, bb), got = md::overlaps(a, b);
        // the same strides: exactly; and from either side alike
        if (want != got || md::overlaps(b, a) != got) { if (bad++ < 10) std::printf("grid %d: %d instead of %d\n", it, got, want); }
        (want ? meet : apart)++;
        const bool extents = md::overlaps(a.p, (size_t)a.extent(0), b.p, (size_t)b.extent(0));
        if (got && !extents) { if (bad++ < 10) std::printf("grid %d: shares a byte outside the extents\n", it); }
        within += extents && !got;
        // other strides: never apart where a byte is shared
        if (axes) {
            const int x = below(axes);
            long other[3] = {stride[0], axes > 1 ? stride[1] : 0, axes > 2 ? stride[2] : 0};
            other[x] += 1 + below(3);
            for (int y = x - 1; y >= 0; --y) if (other[y] < other[y + 1] * nb[y + 1]) other[y] = other[y + 1] * nb[y + 1];
            const md::ByteGrid c = grid(static_cast<const char*>(b.p), axes, other, nb, b.run);
            if (share(ba, bytes(c)) && (!md::overlaps(a, c) || !md::overlaps(c, a))) { if (bad++ < 10) std::printf("grid %d: other strides\n", it); }
            md::ByteGrid f = b;                                              // an axis fewer
            f.axes -= 1;
            for (int y = x; y < f.axes; ++y) { f.stride[y] = b.stride[y + 1]; f.n[y] = b.n[y + 1]; }
            if (share(ba, bytes(f)) && (!md::overlaps(a, f) || !md::overlaps(f, a))) { if (bad++ < 10) std::printf("grid %d: an axis fewer\n", it); }
        }
    }
    if (!(apart > 5000 && meet > 5000 && within > 500)) { std::printf("%ld apart, %ld meet, %ld within extents\n", apart, meet, within); ++bad; }
    md::ByteGrid none = grid(nullptr, 0, nullptr, nullptr, 4);
    if (md::overlaps(none, none)) ++bad;
    if (bad) { std::printf("%d wrong\n", bad); return 1; }
    std::printf("ok\n");
    return 0;
}
