// Queries and keys turned by positions with several axes, and rows turned on their way into the cache held in 4 bits.
//
//   rotate_kernel          rows -> turned rows, q and k in one launch
//   cache4_append_kernel   q -> turned q;  k turned and v as it is -> codes and scales at their slots
//
// Both are bound by memory: six operations to a pair, and each row goes in and out once.
#include "cache4_host.hpp"

namespace md {
namespace {

// Which pair turns by which axis, two bits each.
struct Turn { uint32_t axis[8]; int pairs; };

struct Angles {
    const int32_t *positions, *index;
    const float2* table;
    long plane;                                      // B * L: from axis to axis
    int L, n_pos, axes;
    float sign;                                      // -1: the way back
    Turn turn;
};

// The place of a row on every axis, -1 where it has none.
struct Position { int at[4]; };
__device__ __forceinline__ Position position_of(const Angles& a, int row, int b, int i) {
    const int j = a.index ? a.index[row] : i;
    const bool ok = (uint32_t)j < (uint32_t)a.L;
    Position p;
#pragma unroll
    for (int x = 0; x < 4; ++x) p.at[x] = ok && x < a.axes ? a.positions[x * a.plane + (long)b * a.L + j] : -1;
    return p;
}

// Cosines and sines of pairs p0 .. p0 + W - 1 (p0 a multiple of W, W of 2, 4 or 8; all below `pairs`).
template <int W>
__device__ __forceinline__ void cosines(const Angles& a, const Position& p, int p0, float (&c)[W], float (&s)[W]) {
    uint32_t word = a.turn.axis[0];
#pragma unroll
    for (int x = 1; x < 8; ++x) word = (p0 >> 4) == x ? a.turn.axis[x] : word;
    word >>= 2 * (p0 & 15);
#pragma unroll
    for (int j = 0; j < W; ++j) {
        const int axis = (word >> (2 * j)) & 3;
        int at = p.at[0];
#pragma unroll
        for (int x = 1; x < 4; ++x) at = axis == x ? p.at[x] : at;
        float2 v{__builtin_nanf(""), __builtin_nanf("")};
        if ((uint32_t)at < (uint32_t)a.n_pos) v = a.table[(long)at * a.turn.pairs + p0 + j];
        c[j] = v.x;
        s[j] = v.y * a.sign;
    }
}

// x c - y s and y c + x s: products and sums rounded one by one.
__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
    const float xc = x * c, ys = y * s, yc = y * c, xs = x * s;
    x = xc - ys;
    y = yc + xs;
}

// W channels of a row, as fp32.
template <int W, bool F32>
__device__ __forceinline__ void load_channels(const void* base, long at, float (&x)[W]) {
    if (F32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + at);
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const f32x4 v = p[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
        }
    } else {
        uint32_t w[W / 2];
        if constexpr (W == 8) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
            for (int i = 0; i < W / 2; ++i) w[i] = v[i];
        } else {
            const u32x2 v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
            for (int i = 0; i < W / 2; ++i) w[i] = v[i];
        }
#pragma unroll
        for (int i = 0; i < W / 2; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    }
}
// STREAM: past the caches, for rows by the hundred megabytes.  us: 4 x up to 2371 rows of 64 heads (226 MB in and out) 52.9 with plain stores, 44.0
// so; 16 x up to 777 fp32 rows of 40 + 16 heads of 64 into the cache 38.7 and 34.6.
template <bool STREAM, class V>
__device__ __forceinline__ void put(V v, void* p) {
    if (STREAM) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<V*>(p) = v;
}
template <int W, bool F32, bool STREAM>
__device__ __forceinline__ void store_channels(void* base, long at, const float (&x)[W]) {
    if (F32) {
        float* p = static_cast<float*>(base) + at;
#pragma unroll
        for (int i = 0; i < W / 4; ++i) put<STREAM>(f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]}, p + 4 * i);
    } else {
        uint32_t w[W / 2];
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[i] = as_u32(__builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        if constexpr (W == 8) put<STREAM>(u32x4{w[0], w[1], w[2], w[3]}, p);
        else put<STREAM>(u32x2{w[0], w[1]}, p);
    }
}

// Two runs of W channels of a row that a thread turns, each next to that of the next thread: the halves of pairs p0 .. p0 + W - 1; of neighbours as
// pairs, and of what does not turn, one of the first half of these channels and one of the second.  half: of the row's channels.
template <int W, bool ADJACENT>
struct Runs {
    int c0, c1;
    bool turn0, turn1;
    __device__ __forceinline__ Runs(const Angles& a, int p0, int half) {
        const int pairs = a.turn.pairs;
        turn0 = p0 < (ADJACENT ? 2 * pairs : pairs);
        turn1 = ADJACENT ? p0 + half < 2 * pairs : turn0;
        c0 = ADJACENT || turn0 ? p0 : p0 + pairs;
        c1 = !ADJACENT && turn0 ? p0 + pairs : p0 + half;
    }
    __device__ __forceinline__ void cosines_of(const Angles& a, const Position& pos, float (&c)[W], float (&s)[W]) const {
        if (!ADJACENT) {
            cosines<W>(a, pos, c0, c, s);
            return;
        }
        float c2[W / 2], s2[W / 2];
        cosines<W / 2>(a, pos, c0 / 2, c2, s2);
#pragma unroll
        for (int j = 0; j < W / 2; ++j) { c[j] = c2[j]; s[j] = s2[j]; }
        if (!turn1) return;
        cosines<W / 2>(a, pos, c1 / 2, c2, s2);
#pragma unroll
        for (int j = 0; j < W / 2; ++j) { c[W / 2 + j] = c2[j]; s[W / 2 + j] = s2[j]; }
    }
    __device__ __forceinline__ void turn(const float (&c)[W], const float (&s)[W], float (&lo)[W], float (&hi)[W]) const {
        if (ADJACENT) {
            if (turn0)
#pragma unroll
                for (int j = 0; j < W / 2; ++j) turn_pair(lo[2 * j], lo[2 * j + 1], c[j], s[j]);
            if (turn1)
#pragma unroll
                for (int j = 0; j < W / 2; ++j) turn_pair(hi[2 * j], hi[2 * j + 1], c[W / 2 + j], s[W / 2 + j]);
        } else if (turn0) {
#pragma unroll
            for (int j = 0; j < W; ++j) turn_pair(lo[j], hi[j], c[j], s[j]);
        }
    }
};

// ------------------------------------------------------------------------------------------------ rows

struct Side { const void* x; void* y; KvLayout xl, yl; int heads; };

// A thread turns W pairs (two runs of W channels, or copies as many that do not turn) of HEADS heads of a row: their cosines are read once, and the
// heads' loads are on their way together.  Threads next to each other: channels, then heads.
template <int W, bool F32, bool ADJACENT, int HEADS>
__global__ __launch_bounds__(256) void rotate_kernel(Side q, Side k, Angles ang, const int32_t* __restrict__ rows, int total, FastDiv items,
                                                     FastDiv groups, FastDiv tokens)
{
    const int per = 256 / items.d, slot = items.div(threadIdx.x), item = threadIdx.x - slot * items.d;
    const int u = (int)blockIdx.x * per + slot;      // (the host checks that this fits 31 bits, behind the last one too)
    if (slot >= per || u >= total) return;
    const int row = groups.div(u), g = u - row * groups.d, b = tokens.div(row), i = row - b * tokens.d;
    if (rows && i >= rows[b]) return;
    const Runs<W, ADJACENT> at(ang, item * W, items.d * W);
    float lo[HEADS][W], hi[HEADS][W];
#pragma unroll
    for (int x = 0; x < HEADS; ++x) {
        const int head = g + x * groups.d, of = head - q.heads;
        if (head < q.heads) {
            const long from = (long)b * q.xl.batch + (long)i * q.xl.token + (long)head * q.xl.head;
            load_channels<W, F32>(q.x, from + at.c0, lo[x]);
            load_channels<W, F32>(q.x, from + at.c1, hi[x]);
        } else if (of < k.heads) {
            const long from = (long)b * k.xl.batch + (long)i * k.xl.token + (long)of * k.xl.head;
            load_channels<W, F32>(k.x, from + at.c0, lo[x]);
            load_channels<W, F32>(k.x, from + at.c1, hi[x]);
        }
    }
    float c[W], s[W];
    if (at.turn0) at.cosines_of(ang, position_of(ang, row, b, i), c, s);
#pragma unroll
    for (int x = 0; x < HEADS; ++x) {
        const int head = g + x * groups.d, of = head - q.heads;
        at.turn(c, s, lo[x], hi[x]);
        if (head < q.heads) {
            const long to = (long)b * q.yl.batch + (long)i * q.yl.token + (long)head * q.yl.head;
            store_channels<W, F32, (HEADS > 1)>(q.y, to + at.c0, lo[x]);
            store_channels<W, F32, (HEADS > 1)>(q.y, to + at.c1, hi[x]);
        } else if (of < k.heads) {
            const long to = (long)b * k.yl.batch + (long)i * k.yl.token + (long)of * k.yl.head;
            store_channels<W, F32, (HEADS > 1)>(k.y, to + at.c0, lo[x]);
            store_channels<W, F32, (HEADS > 1)>(k.y, to + at.c1, hi[x]);
        }
    }
}

// ------------------------------------------------------------------------------------------------ rows into the cache

enum { kHalves, kAdjacent, kPart };                  // pairs (i, i + d/2); (2i, 2i + 1); (i, i + pairs) with pairs < d/2

// The channels that a lane's own ones are paired with: where they are halves, those of the lane eight on of sixteen.
template <int D, bool F32, int MODE>
__device__ __forceinline__ void turn_part(const void* base, long row, int part, int pairs, const float (&c)[D / 16], const float (&s)[D / 16],
                                          float (&x)[D / 16]) {
    constexpr int C = D / 16;
    const int at = part * C;
    if (MODE == kAdjacent) {
#pragma unroll
        for (int j = 0; j < C / 2; ++j)
            if (at < 2 * pairs) turn_pair(x[2 * j], x[2 * j + 1], c[j], s[j]);
        return;
    }
    float other[C];
    if (MODE == kHalves) {
#pragma unroll
        for (int j = 0; j < C; ++j) other[j] = dpp_f<0x128>(x[j]);
    } else {
        if (at >= 2 * pairs) return;
        load_part<D, F32>(base, row + (at < pairs ? at + pairs : at - pairs), other);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        float lo = at < pairs ? x[j] : other[j], hi = at < pairs ? other[j] : x[j];
        turn_pair(lo, hi, c[j], s[j]);
        x[j] = at < pairs ? lo : hi;
    }
}

struct Append {
    const void *q, *k, *v;
    void* q_out;
    const int32_t* slots;
    uint8_t* cache;
    KvLayout ql, kl, ol;
    Pool p;
    int Hq, rows, q_blocks;                          // blocks along y that queries take
};

// A wave deals with four rows, sixteen lanes per row with d/16 channels each, of HEADS heads: of the queries, or of K and V.  Blocks next to each
// other: rows, whose codes lie next to each other in a page; where `across` is more than 1, that many blocks of queries with the same rows, whose
// heads lie next to each other.  us with queries by rows / by heads: 16 x 640 rows of 32 + 32 heads of 128 99 / 96.6, of 32 + 8 in fp32 with half of the
// channels turned 107.6 / 88.1, of 32 + 8 in neighbours as pairs 47.3 / 42.3; with K and V by heads, too, 103.7, 85.6, 42.2
template <int D, bool F32, int MODE, int HEADS>
__global__ __launch_bounds__(256) void cache4_append_kernel(Append A, Angles ang, FastDiv tokens, FastDiv across)
{
    constexpr int C = D / 16;
    const int lane = lane_id(), part = lane & 15;
    const bool queries = (int)blockIdx.y < A.q_blocks;
    int rows16 = (int)blockIdx.x, part_of = (int)blockIdx.y;
    if (queries && across.d > 1) {                   // (the host checks that this fits 31 bits)
        const int block = part_of * (int)gridDim.x + rows16;
        rows16 = across.div(block);
        part_of = block - rows16 * across.d;
    }
    const int r = rows16 * 16 + wave_id() * 4 + (lane >> 4);
    C4Slot at{-1, 0};
    if (r < A.rows) at = c4_slot(A.slots[r], A.p.n_pages, A.p.page_shift);
    if (at.page < 0) return;                         // (sixteen lanes together, which are all that exchange anything)
    const int b = tokens.div(r), i = r - b * tokens.d, pairs = ang.turn.pairs;
    const int h0 = (part_of - (queries ? 0 : A.q_blocks)) * HEADS, heads = queries ? A.Hq : A.p.H;
    if constexpr (F32 && D == 128) {                 // (32 bytes to a lane would be half of a line to a store: 88.1 us for the second case above, 77.3 so)
        if (queries) {
            const Runs<4, MODE == kAdjacent> at(ang, part * 4, D / 2);
            const long from = (long)b * A.ql.batch + (long)i * A.ql.token, to = (long)b * A.ol.batch + (long)i * A.ol.token;
            float lo[HEADS][4], hi[HEADS][4], c[4], s[4];
#pragma unroll
            for (int y = 0; y < HEADS; ++y)
                if (h0 + y < heads) {
                    load_channels<4, F32>(A.q, from + (long)(h0 + y) * A.ql.head + at.c0, lo[y]);
                    load_channels<4, F32>(A.q, from + (long)(h0 + y) * A.ql.head + at.c1, hi[y]);
                }
            if (at.turn0) at.cosines_of(ang, position_of(ang, r, b, i), c, s);
#pragma unroll
            for (int y = 0; y < HEADS; ++y)
                if (h0 + y < heads) {
                    at.turn(c, s, lo[y], hi[y]);
                    store_channels<4, F32, (HEADS > 1)>(A.q_out, to + (long)(h0 + y) * A.ol.head + at.c0, lo[y]);
                    store_channels<4, F32, (HEADS > 1)>(A.q_out, to + (long)(h0 + y) * A.ol.head + at.c1, hi[y]);
                }
            return;
        }
    }
    const KvLayout in = queries ? A.ql : A.kl;
    const void* base = queries ? A.q : A.k;
    const long row = (long)b * in.batch + (long)i * in.token;
    float x[HEADS][C] = {}, v[HEADS][C] = {};
#pragma unroll
    for (int y = 0; y < HEADS; ++y)
        if (h0 + y < heads) {
            load_part<D, F32>(base, row + (long)(h0 + y) * in.head + part * C, x[y]);
            if (!queries) load_part<D, F32>(A.v, row + (long)(h0 + y) * in.head + part * C, v[y]);
        }
    float c[C] = {}, s[C] = {};
    if (part * C < 2 * pairs) {
        const Position pos = position_of(ang, r, b, i);
        if (MODE == kAdjacent) {
            float c2[C / 2], s2[C / 2];
            cosines<C / 2>(ang, pos, part * (C / 2), c2, s2);
#pragma unroll
            for (int j = 0; j < C / 2; ++j) { c[j] = c2[j]; s[j] = s2[j]; }
        } else {
            cosines<C>(ang, pos, part * C < pairs ? part * C : part * C - pairs, c, s);
        }
    }
#pragma unroll
    for (int y = 0; y < HEADS; ++y)
        if (h0 + y < heads) turn_part<D, F32, MODE>(base, row + (long)(h0 + y) * in.head, part, pairs, c, s, x[y]);
    if (queries) {
        const long to = (long)b * A.ol.batch + (long)i * A.ol.token + part * C;
#pragma unroll
        for (int y = 0; y < HEADS; ++y)
            if (h0 + y < heads) store_channels<C, F32, (HEADS > 1)>(A.q_out, to + (long)(h0 + y) * A.ol.head, x[y]);
        return;
    }
    const int group = part / (512 / D);
    uint8_t* to = A.cache + ((long)at.page * A.p.H + h0) * A.p.stride;
#pragma unroll
    for (int y = 0; y < HEADS; ++y) {
        int ks, vs;
        const uint32_t kw = quantise_part<D>(x[y], ks), vw = quantise_part<D>(v[y], vs);
        if (h0 + y >= heads) continue;
        store_codes<D>(to + c4_k_codes(at.place, D) + part * (D / 32), kw);
        store_codes<D>(to + c4_v_codes(A.p.page, at.place, part, D), vw);
        if (part % (512 / D) == 0) {
            to[c4_k_scales(A.p.page, at.place, D) + group] = (uint8_t)ks;
            to[c4_v_scales(A.p.page, at.place, group, D)] = (uint8_t)vs;
        }
        to += A.p.stride;
    }
}

// ------------------------------------------------------------------------------------------------ host

int read_rotary(const char* who, const md_rotary* r, int d, int step, int B, int N, int L, int n_pos, const int32_t* positions, const int32_t* index,
                const float* table, int inverse, Angles* out) {
    if (!r || !positions || !table) return fail(MD_EINVAL, "%s: null pointer among the required arguments", who);
    if (L <= 0 || n_pos <= 0) return fail(MD_EINVAL, "%s: L and n_pos must be positive", who);
    if (!index && L < N) return fail(MD_ESHAPE, "%s: positions of %d tokens for %d rows", who, L, N);
    if (r->pairs <= 0 || r->pairs > 128 || r->pairs % step || 2 * r->pairs > d)
        return fail(MD_ESHAPE, "%s: pairs=%d must be a multiple of %d, at most d/2", who, (int)r->pairs, step);
    if (r->axes < 1 || r->axes > 4) return fail(MD_ESHAPE, "%s: axes=%d out of range (1 to 4)", who, (int)r->axes);
    *out = Angles{positions, index, reinterpret_cast<const float2*>(table), (long)B * L, L, n_pos, r->axes, inverse ? -1.f : 1.f, Turn{{}, r->pairs}};
    for (int i = 0; i < r->pairs; ++i) {
        if (r->axis[i] >= r->axes) return fail(MD_EINVAL, "%s: pair %d has axis %d of %d", who, i, (int)r->axis[i], (int)r->axes);
        out->turn.axis[i >> 4] |= (uint32_t)r->axis[i] << (2 * (i & 15));
    }
    if (reinterpret_cast<uintptr_t>(table) & 15u) return fail(MD_EALIGN, "%s: the table must be 16-byte aligned", who);
    return MD_OK;
}
size_t position_bytes(const Angles& a) { return (size_t)a.axes * a.plane * 4; }
size_t table_bytes(const Angles& a) { return (size_t)a.n_pos * a.turn.pairs * 8; }
// An output that is its input, place by place (an axis with one place may have any stride).
bool same_place(const void* x, const KvLayout& l, const void* y, const KvLayout& m, int B, int N, int H) {
    return x == y && (B == 1 || l.batch == m.batch) && (N == 1 || l.token == m.token) && (H == 1 || l.head == m.head);
}

int rotate_impl(const void* q, const void* k, int dtype, const int32_t* positions, const int32_t* index, const float* table, const int32_t* rows,
                int B, int N, int L, int Hq, int H, int d, int n_pos, const md_rotary* rotary, int inverse, void* q_out, void* k_out,
                const md_kv_layout* q_layout, const md_kv_layout* k_layout, const md_kv_layout* q_out_layout, const md_kv_layout* k_out_layout,
                void* stream)
{
    clear_error();
    const char* who = "rotate";
    if (B <= 0 || N <= 0 || Hq <= 0 || d <= 0 || (k && H <= 0)) return fail(MD_EINVAL, "rotate: sizes must be positive");
    if (!q || !q_out || !k != !k_out) return fail(MD_EINVAL, "rotate: null pointer among the required arguments");
    int rc = check_dtype(who, dtype);
    if (rc != MD_OK) return rc;
    if (d % 8 || d > 256) return fail(MD_ESHAPE, "rotate: d=%d must be a multiple of 8, at most 256", d);
    if (Hq > 65535 || (k && H > 65535)) return fail(MD_ESHAPE, "rotate: Hq=%d or H=%d out of range", Hq, H);
    if (!k) H = 0;
    Angles ang;
    rc = read_rotary(who, rotary, d, 4, B, N, L, n_pos, positions, index, table, inverse, &ang);
    Side a{q, q_out, {}, {}, Hq}, c{k, k_out, {}, {}, H};
    if (rc == MD_OK) rc = read_layout(who, "q", q_layout, B, N, Hq, d, &a.xl);
    if (rc == MD_OK) rc = read_layout(who, "q_out", q_out_layout, B, N, Hq, d, &a.yl);
    if (rc == MD_OK && k) rc = read_layout(who, "k", k_layout, B, N, H, d, &c.xl);
    if (rc == MD_OK && k) rc = read_layout(who, "k_out", k_out_layout, B, N, H, d, &c.yl);
    if (rc != MD_OK) return rc;
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(k_out)) return fail(MD_EALIGN, "rotate: tensors must be 16-byte aligned");
    const long all = (long)B * N;
    // loads of 16 bytes, where no pair's halves are split over them.  us for 4 x 2000 fp32 rows of 64 heads, eight
    // channels / four: 120 / 90
    const int W = dtype != MD_F32 && ang.turn.pairs % 8 == 0 && d % 16 == 0 ? 8 : 4, items = d / (2 * W);
    if (all > kMaxRows || all * (Hq + H) * items > 0x7FFFFFFFl - 511) return fail(MD_ESHAPE, "rotate: %ld rows of %d heads are too many for one call", all, Hq + H);
    const ByteGrid qi = rows_grid(q, a.xl, B, N, Hq, d, dtype), qo = rows_grid(q_out, a.yl, B, N, Hq, d, dtype);
    const ByteGrid ki = rows_grid(k, c.xl, B, N, H, d, dtype), ko = rows_grid(k_out, c.yl, B, N, H, d, dtype);
    const Range r[] = {{q_out, rows_bytes(a.yl, B, N, Hq, d, dtype)}, {k_out, k ? rows_bytes(c.yl, B, N, H, d, dtype) : 0}, {positions, position_bytes(ang)},
                       {index, index ? (size_t)all * 4 : 0}, {table, table_bytes(ang)}, {rows, rows ? (size_t)B * 4 : 0}};
    for (int x = 0; x < 2 && rc == MD_OK; ++x) rc = check_apart(who, r[x], r + 2, 4);
    if (rc != MD_OK) return rc;
    if (overlaps(qo, ko) || overlaps(qo, ki) || overlaps(ko, qi) || (!same_place(q, a.xl, q_out, a.yl, B, N, Hq) && overlaps(qo, qi)) ||
        (!same_place(k, c.xl, k_out, c.yl, B, N, H) && overlaps(ko, ki)))
        return fail(MD_EALIAS, "rotate: the outputs and the inputs must not overlap");
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int per = 256 / items;
    // four heads to a thread where there are threads for all of the chip several times over.  us with one / two / four, 4 x up to 2371 rows
    // of 64 heads, plain stores: 62.8 / 55.5 / 52.9
    const bool many = all * (Hq + H) * items >= 4l * 256 * 1024;
    const int groups = many ? (Hq + H + 3) / 4 : Hq + H;
    const int total = (int)(all * groups);
#define MD_ROTATE3(W_, F_, A_, X_)                                                                                                        \
    MD_LAUNCH("rotate", st, (rotate_kernel<W_, F_, A_, X_>), (total + per - 1) / per, 256, 0, a, c, ang, rows, total, FastDiv::make(items), \
        FastDiv::make(groups), FastDiv::make(N))
#define MD_ROTATE2(W_, F_, A_) do { if (many) MD_ROTATE3(W_, F_, A_, 4); else MD_ROTATE3(W_, F_, A_, 1); } while (0)
#define MD_ROTATE(W_, F_) do { if (rotary->adjacent) MD_ROTATE2(W_, F_, true); else MD_ROTATE2(W_, F_, false); } while (0)
    if (dtype == MD_F32) MD_ROTATE(4, true);
    else if (W == 8) MD_ROTATE(8, false);
    else MD_ROTATE(4, false);
#undef MD_ROTATE
#undef MD_ROTATE2
#undef MD_ROTATE3
    return check_launch(who);
}

int append_impl(const void* q, const void* k_new, const void* v_new, int dtype, const int32_t* positions, const int32_t* index, const float* table,
                const int32_t* slots, void* cache, int B, int N, int L, int Hq, int H, int d, int n_pos, int n_pages, int page, const md_rotary* rotary,
                void* q_out, const md_kv_layout* q_layout, const md_kv_layout* rows_layout, const md_kv_layout* q_out_layout, void* stream)
{
    clear_error();
    const char* who = "cache4_append";
    Append A{};
    int rc = check_pool(who, H, d, n_pages, page, 1, &A.p);
    if (rc == MD_OK) rc = check_dtype(who, dtype);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N <= 0 || (q && Hq <= 0)) return fail(MD_EINVAL, "cache4_append: sizes must be positive");
    if (!k_new || !v_new || !slots || !cache || !q != !q_out) return fail(MD_EINVAL, "cache4_append: null pointer among the required arguments");
    if (!q) Hq = 0;
    if (Hq > 65535 - H) return fail(MD_ESHAPE, "cache4_append: Hq=%d and H=%d out of range", Hq, H);
    Angles ang;
    rc = read_rotary(who, rotary, d, 8, B, N, L, n_pos, positions, index, table, 0, &ang);
    if (rc == MD_OK) rc = read_layout(who, "rows", rows_layout, B, N, H, d, &A.kl);
    if (rc == MD_OK && q) rc = read_layout(who, "q", q_layout, B, N, Hq, d, &A.ql);
    if (rc == MD_OK && q) rc = read_layout(who, "q_out", q_out_layout, B, N, Hq, d, &A.ol);
    if (rc != MD_OK) return rc;
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(cache))
        return fail(MD_EALIGN, "cache4_append: tensors must be 16-byte aligned");
    const long rows = (long)B * N;
    if (rows > kMaxRows) return fail(MD_ESHAPE, "cache4_append: %ld rows are too many for one call", rows);
    const size_t in = rows_bytes(A.kl, B, N, H, d, dtype);
    const ByteGrid ki = rows_grid(k_new, A.kl, B, N, H, d, dtype), vi = rows_grid(v_new, A.kl, B, N, H, d, dtype);
    const ByteGrid qi = rows_grid(q, A.ql, B, N, Hq, d, dtype), qo = rows_grid(q_out, A.ol, B, N, Hq, d, dtype);
    const Range r[] = {{cache, pool_bytes(A.p)}, {q_out, q ? rows_bytes(A.ol, B, N, Hq, d, dtype) : 0}, {slots, (size_t)rows * 4}, {positions, position_bytes(ang)},
                       {index, index ? (size_t)rows * 4 : 0}, {table, table_bytes(ang)}, {k_new, in}, {v_new, in}, {q, q ? rows_bytes(A.ql, B, N, Hq, d, dtype) : 0}};
    rc = check_apart(who, r[0], r + 1, 8);
    if (rc == MD_OK) rc = check_apart(who, r[1], r + 2, 4);
    if (rc != MD_OK) return rc;
    if (overlaps(qo, ki) || overlaps(qo, vi) || (!same_place(q, A.ql, q_out, A.ol, B, N, Hq) && overlaps(qo, qi)))
        return fail(MD_EALIAS, "cache4_append: the outputs and the inputs must not overlap");
    A.q = q; A.k = k_new; A.v = v_new; A.q_out = q_out; A.slots = slots; A.cache = static_cast<uint8_t*>(cache); A.Hq = Hq; A.rows = (int)rows;
    hipStream_t st = static_cast<hipStream_t>(stream);
    // two heads to a wave where there are waves for all of the chip more than once.  us with one / two / four, 16 x up to 777 fp32 rows of 40 + 16
    // heads of 64, plain stores: 47.0 / 38.7 / 39.9
    const bool many = (rows + 3) / 4 * (H + Hq) >= 16384;
    const bool by_heads = q && A.ql.head < A.ql.token;
#define MD_C4_APPEND3(D_, F_, M_, X_)                                                                                                     \
    do {                                                                                                                                  \
        A.q_blocks = (Hq + X_ - 1) / X_;                                                                                                  \
        MD_LAUNCH("cache4_append", st, (cache4_append_kernel<D_, F_, M_, X_>), dim3((int)((rows + 15) / 16), A.q_blocks + (H + X_ - 1) / X_), 256, 0, \
            A, ang, FastDiv::make(N), FastDiv::make(by_heads && (rows + 15) / 16 * A.q_blocks < (1L << 31) ? A.q_blocks : 1));             \
    } while (0)
#define MD_C4_APPEND2(D_, F_, M_) do { if (many) MD_C4_APPEND3(D_, F_, M_, 2); else MD_C4_APPEND3(D_, F_, M_, 1); } while (0)
#define MD_C4_APPEND(D_, F_)                                                                                                              \
    do {                                                                                                                                  \
        if (rotary->adjacent) MD_C4_APPEND2(D_, F_, kAdjacent);                                                                           \
        else if (2 * ang.turn.pairs == D_) MD_C4_APPEND2(D_, F_, kHalves);                                                                \
        else MD_C4_APPEND2(D_, F_, kPart);                                                                                                \
    } while (0)
    if (d == 128) { if (dtype == MD_F32) MD_C4_APPEND(128, true); else MD_C4_APPEND(128, false); }
    else { if (dtype == MD_F32) MD_C4_APPEND(64, true); else MD_C4_APPEND(64, false); }
#undef MD_C4_APPEND
#undef MD_C4_APPEND2
#undef MD_C4_APPEND3
    return check_launch(who);
}

}  // namespace
}  // namespace md

extern "C" int mustdrop_rotate(
    const void* q, const void* k, md_dtype dtype, const int32_t* positions, const int32_t* index, const float* table, const int32_t* rows,
    int B, int N, int L, int Hq, int H, int d, int n_pos, const md_rotary* rotary, int inverse, void* q_out, void* k_out,
    const md_kv_layout* q_layout, const md_kv_layout* k_layout, const md_kv_layout* q_out_layout, const md_kv_layout* k_out_layout, void* stream)
{
    return md::rotate_impl(q, k, dtype, positions, index, table, rows, B, N, L, Hq, H, d, n_pos, rotary, inverse, q_out, k_out,
                           q_layout, k_layout, q_out_layout, k_out_layout, stream);
}

extern "C" int mustdrop_cache4_append(
    const void* q, const void* k_new, const void* v_new, md_dtype dtype, const int32_t* positions, const int32_t* index, const float* table,
    const int32_t* slots, void* cache, int B, int N, int L, int Hq, int H, int d, int n_pos, int n_pages, int page, const md_rotary* rotary,
    void* q_out, const md_kv_layout* q_layout, const md_kv_layout* rows_layout, const md_kv_layout* q_out_layout, void* stream)
{
    return md::append_impl(q, k_new, v_new, dtype, positions, index, table, slots, cache, B, N, L, Hq, H, d, n_pos, n_pages, page, rotary,
                           q_out, q_layout, rows_layout, q_out_layout, stream);
}
