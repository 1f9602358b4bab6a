// Attention over a part of the cache held in 4 bits.
//
//   cache4_bounds_kernel          each page's largest and smallest key values, channel by channel, in 8 bits
//   cache4_score_choose_kernel    bounds and queries -> scores in LDS -> the pages to read, for up to 2048 pages and blocks enough
//   cache4_score_kernel           bounds and queries -> a score for each token, K/V head and page
//   cache4_choose_block_kernel    scores -> the pages to read, for up to 8192 of them, in registers
//   cache4_choose_kernel          the same for any number, which it looks up again and again
//   cache4_attend_chosen_kernel   softmax(scale Q K^T) V over them
//   cache4_attend_shared_kernel   the same for several tokens together, over all of their pages
//   cache4_attend_chosen_join_kernel   what parts of a list have given, put together
//
// The score of a page is the sum over the G query heads of max over [smallest, largest] of q . k, which is no less than the sum of any of its
// keys' own scores: max(q a, q b) = max(q, 0) a + min(q, 0) b for a >= b, so that it is one matrix product with twice the channels.
// Bounds and queries are whole numbers of 8 bits times a power of two: their sums are exact, whatever the order, and so is the choice.
#include "cache4_host.hpp"

namespace md {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------------ bounds

// Of 2 S numbers S: maxima over lanes that differ in bit BIT; lanes with the bit set go on with the upper half, the others with the lower.
template <int BIT, int S>
__device__ __forceinline__ void halve(float (&v)[16], int lane) {
#pragma unroll
    for (int c = 0; c < S; ++c) {
        uint32_t x = __float_as_uint(v[c]), y = __float_as_uint(v[c + S]);
        if constexpr (BIT == 8) {
            const bool up = lane & 8;
            const uint32_t give = up ? x : y;
            x = up ? y : x;
            y = (uint32_t)dpp_i<0x128>((int)give, (int)give);
        } else {                                     // the two registers change halves: one instruction
            const auto r = BIT == 32 ? __builtin_amdgcn_permlane32_swap(x, y, false, false) : __builtin_amdgcn_permlane16_swap(x, y, false, false);
            x = r[0];
            y = r[1];
        }
        v[c] = fmaxf(__uint_as_float(x), __uint_as_float(y));
    }
}

// A wave per page and head.  Sixteen (d = 64: eight) lanes side by side have the channels of one token, eight each: of all tokens they keep the
// largest values and the largest with the sign turned, 16 numbers.  The four (eight) lanes of the same channels then halve these among
// them until each has 4 (2) of the one kind, which is a word (half of one) of the result.  (Sixteen bytes to a lane are fewer loads, but 64
// numbers to halve over sixteen lanes: 22 us for the bounds of 16 x up to 5888 entries of 8 heads instead of 10.6.)
// AHEAD: tokens of a lane that are on their way together, eight, or as many as a small page has: what follows the loads bounds
// these.  us with eight / so, 16 x up to 5888 entries of 8 heads: d = 64, pages of 16 27.6 / 17.6, of 32 15.1 / 11.9; d = 128, of 16 27.6 / 21.3
template <int D, int AHEAD>
__global__ __launch_bounds__(256) void cache4_bounds_kernel(
    const uint8_t* __restrict__ cache, const int32_t* __restrict__ table, const int32_t* __restrict__ len, const int32_t* __restrict__ first,
    int8_t* __restrict__ bounds, uint8_t* __restrict__ scales, Pool p, int units, int N, FastDiv heads, FastDiv span)
{
    constexpr int PARTS = D / 8, TOKENS = kWave / PARTS;
    const int unit = (int)blockIdx.x * 4 + wave_id(), lane = lane_id();
    if (unit >= units) return;
    const int bx = heads.div(unit), h = unit - bx * heads.d, b = span.div(bx), x = bx - b * span.d;
    int length = uniform(len)[b], from = uniform(first ? first : len)[b];
    asm volatile("" : "+s"(length), "+s"(from));     // (on their way together)
    length = c4_clamp(length, 0, p.max_pages << p.page_shift);
    from = first ? max(from, 0) : 0;
    const long e = (long)(from >> p.page_shift) + x, stop = min((long)from + N, (long)length);
    if (from >= stop || (e << p.page_shift) >= stop) return;                 // (the page of an entry that is not there yet may hold others)
    const int id = c4_page_id(table[(long)b * p.max_pages + e], p.n_pages);
    if (id < 0) return;
    const int live = min(length - (int)(e << p.page_shift), p.page);
    const uint8_t* base = cache + ((long)id * p.H + h) * p.stride;
    const int part = lane & (PARTS - 1), t0 = lane / PARTS;
    float v[16];                                     // largest, then largest of the negative, of 8 channels
#pragma unroll
    for (int c = 0; c < 16; ++c) v[c] = -INFINITY;
    uint32_t top = 0;                                // the largest scale
    for (int t = t0; t - t0 < live; t += TOKENS * AHEAD) {
        uint32_t w[AHEAD], code[AHEAD];
#pragma unroll
        for (int y = 0; y < AHEAD; ++y) {     // (the last token in the place of those behind it)
            const int at = min(t + y * TOKENS, live - 1);
            w[y] = *reinterpret_cast<const uint32_t*>(base + c4_k_codes(at, D) + part * 4);
            code[y] = base[c4_k_scales(p.page, at, D) + part / 4];
        }
#pragma unroll
        for (int y = 0; y < AHEAD; y += 2) {
            const float s = scale_of(code[y]), s2 = scale_of(code[y + 1]);
            top = max(top, max(code[y], code[y + 1]));
            const f32x2 a[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y], s, 1),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y], s, 3)};
            const f32x2 z[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y + 1], s2, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y + 1], s2, 1),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y + 1], s2, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[y + 1], s2, 3)};
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float f = a[c >> 1][c & 1], g = z[c >> 1][c & 1];
                asm("v_max3_f32 %0, %0, %1, %2" : "+v"(v[c]) : "v"(f), "v"(g));
                asm("v_max3_f32 %0, %0, -%1, -%2" : "+v"(v[8 + c]) : "v"(f), "v"(g));
            }
        }
    }
    halve<32, 8>(v, lane);
    halve<16, 4>(v, lane);
    if (D == 64) halve<8, 2>(v, lane);
    constexpr int LEFT = D == 128 ? 4 : 2;
    float most = v[0];
#pragma unroll
    for (int c = 1; c < LEFT; ++c) most = fmaxf(most, v[c]);
    most = wave_max(most);                           // the largest magnitude: of a channel's largest and smallest value one has it
    const bool none = __any(top >= 253);             // (6 * 2^126 is no number of fp32)
    const int ex = most > 0.f ? max((int)(__float_as_uint(most) >> 23) - 127 - 6, -126) : -126;
    const bool least = lane & 32;
    uint32_t word = 0;
#pragma unroll
    for (int c = 0; c < LEFT; ++c) {
        const int up = none ? 0 : (int)ceilf(__builtin_amdgcn_ldexpf(v[c], -ex));
        word |= (uint32_t)((least ? -up : up) & 0xFF) << (8 * c);
    }
    const int channel = part * 8 + (lane & 16 ? 4 : 0) + (D == 64 && (lane & 8) ? 2 : 0);
    int8_t* to = bounds + ((long)id * p.H + h) * (2 * D) + (least ? D : 0) + channel;
    if (D == 128) *reinterpret_cast<uint32_t*>(to) = word;
    else *reinterpret_cast<uint16_t*>(to) = (uint16_t)word;
    if (lane == 0) scales[(long)id * p.H + h] = none ? 255 : (uint8_t)(ex + 127);
}

// ------------------------------------------------------------------------------------------------ scores

struct Choose {
    const void* q;
    const int8_t* bounds;
    const uint8_t* scales;
    const int32_t *table, *len, *q_len;
    int32_t* chosen;
    float* scores;                                   // [B, H, N, pitch]
    KvLayout ql;
    int B, N, G, H, n_pages, max_pages, page_shift, pitch;
    int first, last, budget;
    int lanes, subs, per, tiles;                     // query heads of a token side by side (a power of two), tiles of them, tokens of a tile, tiles of tokens
    bool together;                                   // (what the host goes by)
    size_t lds;
};

// Pages that row i of sample b sees; -1 where there is no such row.
__device__ __forceinline__ int pages_seen(const Choose& A, int b, int i) {
    const int length = c4_clamp(A.len[b], 0, A.max_pages << A.page_shift), nq = A.q_len ? c4_clamp(A.q_len[b], 0, A.N) : A.N;
    if (i >= nq) return -1;
    return c4_pages_of(min(max(length - nq + i + 1, 0), length), A.page_shift);
}

// W channels of a query as they lie in memory.
template <int W, bool F32>
struct Raw {
    static constexpr int WORDS = F32 ? W : W / 2;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const void* base, long at) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
        if constexpr (WORDS == 2) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(p);
            w[0] = v[0];
            w[1] = v[1];
        } else {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
            }
        }
    }
    __device__ __forceinline__ float at(int j) const { return F32 ? __uint_as_float(w[j]) : j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]); }
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) m = max(m, __float_as_uint(at(j)) & 0x7FFFFFFFu);
        return m;
    }
    // Their whole numbers as bytes: those above 0, and those below with their sign turned.  (The hardware's conversion to a byte takes what
    // is below 0 as 0.)
    __device__ __forceinline__ void whole(int shift, uint32_t ok, uint32_t (&above)[W / 4], uint32_t (&below)[W / 4]) const {
#pragma unroll
        for (int x = 0; x < W / 4; ++x) {
            uint32_t a = 0, b = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float n = __builtin_amdgcn_fmed3f(__builtin_rintf(__builtin_amdgcn_ldexpf(at(4 * x + j), shift)), -127.f, 127.f);
                a = __builtin_amdgcn_cvt_pk_u8_f32(n, j, a);
                b = __builtin_amdgcn_cvt_pk_u8_f32(-n, j, b);
            }
            above[x] = a & ok;
            below[x] = b & ok;
        }
    }
};
// The step of numbers whose largest magnitude has these bits, as a shift; and whether they count at all.
__device__ __forceinline__ int whole_shift(uint32_t most) { return 7 - __builtin_amdgcn_frexp_expf(__uint_as_float(most)); }
__device__ __forceinline__ uint32_t whole_ok(uint32_t most) { return most > 0 && most < 0x7F800000u ? ~0u : 0u; }

// Of lanes side by side, `lanes` (a power of two up to 16) of them: the largest, the sum.  `m`: all ones for as many steps as that takes.
struct Steps {
    uint32_t m[4];
    __device__ __forceinline__ explicit Steps(int lanes) {
#pragma unroll
        for (int x = 0; x < 4; ++x) m[x] = lanes > 1 << x ? ~0u : 0u;
    }
    __device__ __forceinline__ uint32_t largest(uint32_t v) const {
        v = max(v, (uint32_t)dpp_i<0xB1>((int)v, (int)v) & m[0]);
        v = max(v, (uint32_t)dpp_i<0x4E>((int)v, (int)v) & m[1]);
        v = max(v, (uint32_t)dpp_i<0x141>((int)v, (int)v) & m[2]);
        return max(v, (uint32_t)dpp_i<0x140>((int)v, (int)v) & m[3]);
    }
    __device__ __forceinline__ int sum(int v) const {
        v += dpp_i<0xB1>(v, v) & (int)m[0];
        v += dpp_i<0x4E>(v, v) & (int)m[1];
        v += dpp_i<0x141>(v, v) & (int)m[2];
        return v + (dpp_i<0x140>(v, v) & (int)m[3]);
    }
};

// 16 query rows (the G heads of some tokens, filled up with zeros to a power of two; MULTI, more than 16 heads: one 16 after the other) against
// T tiles of 16 pages at a time, by a wave of a block of 256 threads.  Lane (n, lb) has bytes lb * 16 .. + 15 of every 64 of row n of either
// operand.  A block's waves turn the queries into whole numbers together and share them through LDS (each for itself: 64 x up to 4096 entries
// of 32 heads 13.2 us instead of 12.3); MULTI: each for itself.
// There are few instructions to a byte, and nothing else to do while a wave waits: what does not depend on the sample's length is asked for
// together with it, and nothing is loaded under a condition of a lane (rows and pages that are not there are others' in their place, and
// count as nothing).
template <int D, bool F32, bool MULTI, int T>
struct Scorer {
    static constexpr int Y = D / 64, W = D / 16, PITCH = D + 16;     // channels of a thread's share; bytes of a row in LDS
    static constexpr int LDS = 16 * 4 + 2 * 16 * PITCH;
    const Choose& A;
    Steps steps;
    int b, h, tile, i, g0, n, lb, length, nq;
    Raw<W, F32> share;                               // of row threadIdx.x / 16
    int entry[T], mine[T];                           // of the block table, for the tiles that come next: of page n, and of 4 lb + n % 4
    i32x4 above[Y], below[Y], hi[T][Y], lo[T][Y];
    int code[T];                                     // of page 4 lb + n % 4 in each tile: its scale; 256: no page

    __device__ __forceinline__ Scorer(const Choose& A_, int b_, int h_, int tile_, int first) : A(A_), steps(A_.lanes), b(b_), h(h_), tile(tile_) {
        const int lane = lane_id();
        n = lane & 15;
        lb = lane >> 4;
        i = tile * A.per + n / A.lanes;
        g0 = n & (A.lanes - 1);
        length = uniform(A.len)[b];
        nq = uniform(A.q_len ? A.q_len : A.len)[b];
        if (!MULTI) share.load(A.q, query_at((int)threadIdx.x >> 4, 0) + (threadIdx.x & 15) * W);
        ask(first);
        asm volatile("" : "+s"(length), "+s"(nq));   // (asked for here, and not where a condition lets them)
#pragma unroll
        for (int t = 0; t < T; ++t) asm volatile("" : "+v"(entry[t]), "+v"(mine[t]));
        length = c4_clamp(length, 0, A.max_pages << A.page_shift);
        nq = A.q_len ? c4_clamp(nq, 0, A.N) : A.N;
    }
    // Pages that row `row` sees.
    __device__ __forceinline__ int seen_by(int row) const { return c4_pages_of(min(max(length - nq + row + 1, 0), length), A.page_shift); }
    // Where a row's query begins, or another one's where there is no such row.
    __device__ __forceinline__ long query_at(int row, int sub) const {
        const int token = min(tile * A.per + row / A.lanes, A.N - 1), g = min(sub * 16 + (row & (A.lanes - 1)), A.G - 1);
        return (long)b * A.ql.batch + (long)token * A.ql.token + (long)(h * A.G + g) * A.ql.head;
    }
    __device__ __forceinline__ bool there(int row, int sub) const { return tile * A.per + row / A.lanes < nq && sub * 16 + (row & (A.lanes - 1)) < A.G; }

    __device__ __forceinline__ void ask(int first) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int32_t* row = A.table + (long)b * A.max_pages;
            entry[t] = row[min((first + t) * 16 + n, A.max_pages - 1)];
            mine[t] = row[min((first + t) * 16 + 4 * lb + (n & 3), A.max_pages - 1)];
        }
    }
    // Bounds of the tiles whose entries have been asked for, on their way; then the entries of tiles next ..
    __device__ __forceinline__ void fetch(int next) {
        const auto page = [&](int e) { return (long)((uint32_t)e < (uint32_t)A.n_pages ? e : 0) * A.H + h; };
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int8_t* from = A.bounds + page(entry[t]) * (2 * D) + lb * 16;
            code[t] = A.scales[page(mine[t])] | ((uint32_t)mine[t] < (uint32_t)A.n_pages ? 0 : 256);
#pragma unroll
            for (int y = 0; y < Y; ++y) {
                hi[t][y] = *reinterpret_cast<const i32x4*>(from + y * 64);
                lo[t][y] = *reinterpret_cast<const i32x4*>(from + D + y * 64);
            }
        }
        ask(next);
        __builtin_amdgcn_sched_barrier(0);
    }
    // The queries' whole numbers: by all of the block, or by the wave for itself.  `lds`: LDS bytes.
    __device__ __forceinline__ void queries(char* lds) {
        uint32_t* s_most = reinterpret_cast<uint32_t*>(lds);
        char* s_whole = lds + 64;
        const int row = (int)threadIdx.x >> 4, part = threadIdx.x & 15;
        uint32_t most = there(row, 0) ? share.largest() : 0u;
        most = Steps(16).largest(most);
        if (part == 0) s_most[row] = most;
        block_sync_lds();
        most = steps.largest(s_most[n]);
        most = (uint32_t)__shfl((int)most, row & 15, kWave);
        uint32_t a[W / 4], c[W / 4];
        share.whole(whole_shift(most), there(row, 0) ? whole_ok(most) : 0u, a, c);
        uint32_t* to = reinterpret_cast<uint32_t*>(s_whole + row * PITCH + part * W);
#pragma unroll
        for (int x = 0; x < W / 4; ++x) { to[x] = a[x]; to[16 * PITCH / 4 + x] = c[x]; }
        block_sync_lds();
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            above[y] = *reinterpret_cast<const i32x4*>(s_whole + n * PITCH + lb * 16 + y * 64);
            below[y] = *reinterpret_cast<const i32x4*>(s_whole + (16 + n) * PITCH + lb * 16 + y * 64);
        }
    }
    __device__ __forceinline__ void multiply(i32x4 (&up)[T], i32x4 (&down)[T]) const {
#pragma unroll
        for (int y = 0; y < Y; ++y)
#pragma unroll
            for (int t = 0; t < T; ++t) {
                up[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi[t][y], above[y], up[t], 0, 0, 0);
                down[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(lo[t][y], below[y], down[t], 0, 0, 0);
            }
    }
    __device__ __forceinline__ void multiply_many(i32x4 (&up)[T], i32x4 (&down)[T]) {
        Raw<16, F32> x;
        uint32_t most = 0;
        for (int s = 0; s < A.subs; ++s)
            for (int y = 0; y < Y; ++y) {
                x.load(A.q, query_at(n, s) + lb * 16 + y * 64);
                most = max(most, there(n, s) ? x.largest() : 0u);
            }
        most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32, kWave));
        most = steps.largest(most);
        for (int s = 0; s < A.subs; ++s) {
#pragma unroll
            for (int y = 0; y < Y; ++y) {
                uint32_t a[4], c[4];
                x.load(A.q, query_at(n, s) + lb * 16 + y * 64);
                x.whole(whole_shift(most), there(n, s) ? whole_ok(most) : 0u, a, c);
                above[y] = i32x4{(int)a[0], (int)a[1], (int)a[2], (int)a[3]};
                below[y] = i32x4{(int)c[0], (int)c[1], (int)c[2], (int)c[3]};
            }
            multiply(up, down);
        }
    }

    // Scores of the pages of tiles first .. first + T - 1 (below `seen`), whose bounds have been fetched: each(token, page, four scores), by one
    // lane of a token's and for four pages at a time.
    template <class Each>
    __device__ __forceinline__ void score(int first, int seen, Each each) {
        i32x4 up[T] = {}, down[T] = {};
        if (MULTI) multiply_many(up, down);
        else multiply(up, down);
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int e0 = (first + t) * 16 + 4 * lb;                // up[t][x]: page e0 + x, query n
            i32x4 sum = up[t] - down[t];
            if (A.lanes > 1) {
#pragma unroll
                for (int x = 0; x < 4; ++x) sum[x] = steps.sum(sum[x]);
            }
            const int c[4] = {dpp_i<0x00>(code[t], code[t]), dpp_i<0x55>(code[t], code[t]), dpp_i<0xAA>(code[t], code[t]), dpp_i<0xFF>(code[t], code[t])};
            f32x4 score;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float v = __builtin_amdgcn_ldexpf((float)sum[x], c[x] - 127);
                score[x] = c[x] < 255 ? v : c[x] == 255 ? INFINITY : -INFINITY;
            }
            if (i < nq && g0 == 0 && e0 < seen) each(i, e0, score);
        }
    }
};

// Scores into the workspace: a wave takes kScoreTiles tiles of pages.
constexpr int kScoreTiles = 2;
template <int D, bool F32, bool MULTI>
__global__ __launch_bounds__(256, 4) void cache4_score_kernel(Choose A, FastDiv tiles, FastDiv heads)
{
    typedef Scorer<D, F32, MULTI, kScoreTiles> S;
    __shared__ f32x4 s_lds[MULTI ? 1 : S::LDS / 16];
    const int bh = tiles.div(blockIdx.x), tile = blockIdx.x - bh * tiles.d, b = heads.div(bh), h = bh - b * heads.d;
    const int first = ((int)blockIdx.y * 4 + wave_id()) * kScoreTiles;
    S sc(A, b, h, tile, first);
    if (tile * A.per >= sc.nq) return;
    const int seen = sc.seen_by(min(sc.nq, (tile + 1) * A.per) - 1);
    if ((int)blockIdx.y * 4 * kScoreTiles * 16 >= seen) return;
    sc.fetch(first);
    if (!MULTI) sc.queries(reinterpret_cast<char*>(s_lds));
    sc.score(first, seen, [&](int i, int e0, f32x4 score) {
        *reinterpret_cast<f32x4*>(A.scores + ((long)bh * A.N + i) * A.pitch + e0) = score;
    });
}

// ------------------------------------------------------------------------------------------------ choice

// A score as a whole number of the same order; above 0, and below all ones.
__device__ __forceinline__ uint32_t ordered(float score) {
    const uint32_t u = __float_as_uint(score + 0.f);     // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Where the chosen scores end: those above `bound`, and the first `ties` of those equal to it.
struct Border { uint32_t bound; int ties; };
// The border of the `need` largest of the keys that lanes have with a bit in `ranked` (there are more), all between `least` and `most`: by histograms
// of eight bits from the first one on that differs, until a place of one is taken whole.  By a wave (hist: 256 ints of its own) or by a
// block of 256 threads (4 x 256 ints, zeros).  us for 64 of up to 1563 scores, 80 times, a block each: 5.4; with votes instead, for two bits at
// a time, 8.8.
template <int K, bool BLOCK>
__device__ __forceinline__ Border border_of(const uint32_t (&key)[K], uint32_t ranked, int need, uint32_t least, uint32_t most, int* hist) {
    if (need <= 0) return Border{0xFFFFFFFEu, 0};
    const int lane = lane_id(), from = 31 - __clz((int)((least ^ most) | 1u));
    uint32_t bound = (most >> from >> 1) << 1 << from, width = 0xFFFFFFFFu >> (31 - from);       // (the width less one)
    for (int sh = max(from - 7, 0);; sh = max(sh - 8, 0)) {
        if (!BLOCK) reinterpret_cast<i32x4*>(hist)[lane] = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (((ranked >> j) & 1) && key[j] - bound <= width) atomicAdd(&hist[(key[j] - bound) >> sh], 1);
        if (BLOCK) block_sync_lds();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        // places 255, 254, .. by four to a lane
        const i32x4 c = reinterpret_cast<const i32x4*>(hist)[kWave - 1 - lane];
        const int sum = (c[3] + c[2]) + (c[1] + c[0]), upto = wave_incl_scan_i(sum);
        int before = upto - sum, place = -1, left = 0, in = 0;
#pragma unroll
        for (int x = 3; x >= 0; --x) {
            if (before < need && before + c[x] >= need) { place = 4 * (kWave - 1 - lane) + x; left = need - before; in = c[x]; }
            before += c[x];
        }
        const int at = (int)__builtin_ctzll(__ballot(place >= 0));
        place = __builtin_amdgcn_readlane(place, at);
        need = __builtin_amdgcn_readlane(left, at);
        in = __builtin_amdgcn_readlane(in, at);
        bound += (uint32_t)place << sh;
        if (need == in) return Border{bound - 1, 0};             // (a key is never 0, and so is no bound that is taken whole)
        if (sh == 0) return Border{bound, need};
        width = (1u << sh) - 1;
        if (BLOCK) hist += 256;
    }
}

// The choice by one wave, whose lane l has the scores of pages l, l + 64, .. in registers.
template <int K>
__device__ __forceinline__ void choose_by_wave(const Choose& A, const float* score, int P, int32_t* to, int* hist) {
    const int lane = lane_id(), hi = P - A.last, taken = A.budget;
    if (P <= A.budget) {
        for (int x = lane; x < A.budget; x += kWave) to[x] = x < P ? x : -1;
        return;
    }
    uint32_t key[K], least = 0xFFFFFFFFu, most = 0, ranked = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int e = j * kWave + lane;
        const bool in = e >= A.first && e < hi;
        key[j] = in ? ordered(score[e]) : e < P ? 0xFFFFFFFFu : 0u;
        least = min(least, in ? key[j] : 0xFFFFFFFFu);
        most = max(most, in ? key[j] : 0u);
        ranked |= in ? 1u << j : 0u;
    }
    const Border r = border_of<K, false>(key, ranked, taken - A.first - A.last, wave_min_u32(least), ~wave_min_u32(~most), hist);
    int done = 0, ties = r.ties;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (j * kWave >= P) break;
        const unsigned long long same = __ballot(ties > 0 && key[j] == r.bound);
        const bool in = key[j] > r.bound || (ties > 0 && key[j] == r.bound && lanes_below(same) < ties);
        ties -= (int)__popcll(same);
        const unsigned long long on = __ballot(in);
        if (in) to[done + lanes_below(on)] = j * kWave + lane;
        done += (int)__popcll(on);
    }
}

// Scores and choice in one: a block per tile of 16 query rows, scores in LDS ([tokens][pitch]), a wave per token for the choice.
template <int D, bool F32, int K>
__global__ __launch_bounds__(256, 4) void cache4_score_choose_kernel(Choose A, FastDiv tiles, FastDiv heads)
{
    extern __shared__ f32x4 s_lds[];
    __shared__ __align__(16) int s_hist[4][256];
    float* s_score = reinterpret_cast<float*>(s_lds);
    const int bh = tiles.div(blockIdx.x), tile = blockIdx.x - bh * tiles.d, b = heads.div(bh), h = bh - b * heads.d;
    const int i0 = tile * A.per, waves = blockDim.x >> 6;
    int first = wave_id() * kScoreTiles;
    typedef Scorer<D, F32, false, kScoreTiles> S;
    S sc(A, b, h, tile, first);
    if (i0 >= sc.nq) return;
    const int last = min(sc.nq, i0 + A.per) - 1, seen = sc.seen_by(last);
    if (seen > A.budget) {
        sc.fetch(first + waves * kScoreTiles);
        sc.queries(reinterpret_cast<char*>(s_lds));
        s_score += S::LDS / 4;
        while (first * 16 < seen) {
            sc.score(first, seen, [&](int i, int e0, f32x4 score) {
                *reinterpret_cast<f32x4*>(s_score + (i - i0) * A.pitch + e0) = score;
            });
            first += waves * kScoreTiles;
            if (first * 16 < seen) sc.fetch(first + waves * kScoreTiles);
        }
        __syncthreads();
    }
    for (int i = i0 + wave_id(); i <= last; i += waves)
        choose_by_wave<K>(A, s_score + (i - i0) * A.pitch, sc.seen_by(i), A.chosen + (((long)b * A.N + i) * A.H + h) * A.budget, s_hist[wave_id()]);
}

// The list that a block deals with, of one launch's rows of blocks (c4_lists); -1 behind the last one.
__device__ __forceinline__ int list_at(const Choose& A) {
    const uint32_t at = blockIdx.y * gridDim.x + blockIdx.x;             // (fewer than 2^23 + 2^21)
    return at < (uint32_t)(A.B * A.H * A.N) ? (int)at : -1;
}

// The same by the waves of a block, of up to WAVES * 512 scores in the workspace: wave w's lane l has those of pages (WAVES j + w) * 64 + l.
template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void cache4_choose_block_kernel(Choose A, FastDiv tokens, FastDiv heads)
{
    constexpr int K = 8, PER = WAVES * K / kWave < 1 ? 1 : WAVES * K / kWave;       // counts of 64 pages to a lane
    __shared__ __align__(16) int s_hist[4 * 256];
    __shared__ uint32_t s_least[WAVES], s_most[WAVES];
    __shared__ int s_count[WAVES * K];
    const int list = list_at(A);
    if (list < 0) return;
    const int bh = tokens.div(list), i = list - bh * tokens.d, b = heads.div(bh), h = bh - b * heads.d;
    const int lane = lane_id(), wv = wave_id();
    const float* score = A.scores + (long)list * A.pitch;
    float f[K];
#pragma unroll
    for (int j = 0; j < K; ++j) f[j] = score[min((WAVES * j + wv) * kWave + lane, A.pitch - 1)];     // (on their way with the length)
    int length = uniform(A.len)[b], nq = uniform(A.q_len ? A.q_len : A.len)[b];
    asm volatile("" : "+s"(length), "+s"(nq));
#pragma unroll
    for (int j = 0; j < K; ++j) asm volatile("" : "+v"(f[j]));
    length = c4_clamp(length, 0, A.max_pages << A.page_shift);
    nq = A.q_len ? c4_clamp(nq, 0, A.N) : A.N;
    if (i >= nq) return;
    const int P = c4_pages_of(min(max(length - nq + i + 1, 0), length), A.page_shift), hi = P - A.last, taken = A.budget;
    int32_t* to = A.chosen + (((long)b * A.N + i) * A.H + h) * A.budget;
    if (P <= taken) {
        for (int x = threadIdx.x; x < taken; x += WAVES * 64) to[x] = x < P ? x : -1;
        return;
    }
    uint32_t key[K], least = 0xFFFFFFFFu, most = 0, ranked = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int e = (WAVES * j + wv) * kWave + lane;
        const bool in = e >= A.first && e < hi;
        key[j] = in ? ordered(f[j]) : e < P ? 0xFFFFFFFFu : 0u;
        least = min(least, in ? key[j] : 0xFFFFFFFFu);
        most = max(most, in ? key[j] : 0u);
        ranked |= in ? 1u << j : 0u;
    }
    least = wave_min_u32(least);
    most = ~wave_min_u32(~most);
    if (lane == 0) { s_least[wv] = least; s_most[wv] = most; }
    if (threadIdx.x < 256) reinterpret_cast<i32x4*>(s_hist)[threadIdx.x] = i32x4{0, 0, 0, 0};
    block_sync_lds();
    least = wave_min_u32(s_least[lane & (WAVES - 1)]);
    most = ~wave_min_u32(~s_most[lane & (WAVES - 1)]);
    const Border r = border_of<K, true>(key, ranked, taken - A.first - A.last, least, most, s_hist);
    // larger ones and equal ones of 64 at a time, and before them
    int mine[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        mine[j] = (int)__popcll(__ballot(key[j] > r.bound)) | (r.ties ? (int)__popcll(__ballot(key[j] == r.bound)) << 16 : 0);
        if (lane == 0) s_count[WAVES * j + wv] = mine[j];
    }
    block_sync_lds();
    int count[PER], sum = 0;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        count[x] = lane * PER + x < WAVES * K ? s_count[lane * PER + x] : 0;
        sum += count[x];
    }
    const int upto = wave_incl_scan_i(sum), behind = PER == 2 ? count[PER - 1] : 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int at = WAVES * j + wv;               // (of the two of a lane, the first one has the second behind it)
        const int before = __builtin_amdgcn_readlane(upto, at / PER) - (PER == 2 && !(at & 1) ? __builtin_amdgcn_readlane(behind, at / PER) : 0) - mine[j];
        const bool larger = key[j] > r.bound, same = r.ties && key[j] == r.bound;
        const int equal = (before >> 16) + lanes_below(__ballot(same));
        if (larger || (same && equal < r.ties)) to[(before & 0xFFFF) + lanes_below(__ballot(larger)) + min(equal, r.ties)] = (WAVES * j + wv) * kWave + lane;
    }
}

// Larger scores first, of equal ones the first page; never 0.
__device__ __forceinline__ uint64_t page_key(float score, int e) { return ((uint64_t)ordered(score) << 32) | (uint32_t)(0x7FFFFFFF - e); }

// The choice from any number of scores in the workspace, a block per token and K/V head, which looks them up again and again.
__global__ __launch_bounds__(1024) void cache4_choose_kernel(Choose A, FastDiv tokens, FastDiv heads)
{
    __shared__ int s_hist[kSelectHistInts], s_red[16];
    const int list = list_at(A);
    if (list < 0) return;
    const int bh = tokens.div(list), i = list - bh * tokens.d, b = heads.div(bh), h = bh - b * heads.d, tid = threadIdx.x;
    const int P = pages_seen(A, b, i);
    if (P < 0) return;
    const float* score = A.scores + (long)list * A.pitch;
    int32_t* to = A.chosen + (((long)b * A.N + i) * A.H + h) * A.budget;
    if (P <= A.budget) {
        for (int x = tid; x < A.budget; x += 1024) to[x] = x < P ? x : -1;
        return;
    }
    const int lo = A.first, hi = P - A.last, always = lo + P - hi;       // pages lo .. hi - 1 are ranked
    for (int x = tid; x < kSelectHistInts; x += 1024) s_hist[x] = 0;
    __syncthreads();
    const SelectBound bound = block_select_keys([&](auto f) {
        for (int e = lo + tid; e < hi; e += 1024) f(page_key(score[e], e));
    }, A.budget - always, s_hist);
    int done = 0;
    for (int e0 = 0; e0 < P; e0 += 1024) {
        const int e = e0 + tid;
        const bool in = e < P && (e < lo || e >= hi || (A.budget > always && (page_key(score[e], e) >> bound.shift) >= bound.bound));
        int total;
        const int at = block_rank(in, s_red, total);
        if (in && done + at < A.budget) to[done + at] = e;
        done += total;
    }
}

// ------------------------------------------------------------------------------------------------ attention

// A walk over the pages of a list, which lies in LDS: page numbers and entries of the block table.  Positions of the walk count the
// list's tokens, one page after the other.
struct Listed : Walk {
    uint32_t list;                                   // in LDS
    int last;                                        // of the list
};
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_ptr_t)const_cast<void*>(p); }
// Of a step's two 16-key tiles (to the compiler a read of LDS is one of what the loads on their way write there, and would wait for them all)
struct Entries { int id[2], entry[2]; };
__device__ __forceinline__ Entries listed_at(const Listed& w, int step) {
    u32x2 a, b;
    asm volatile("ds_read_b64 %0, %2\n\tds_read_b64 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(a), "=&v"(b)
                 : "v"(w.list + 8 * min((step * 32) >> w.page_shift, w.last)), "v"(w.list + 8 * min((step * 32 + 16) >> w.page_shift, w.last)) : "memory");
    return Entries{{__builtin_amdgcn_readfirstlane((int)a.x), __builtin_amdgcn_readfirstlane((int)b.x)},
                   {__builtin_amdgcn_readfirstlane((int)a.y), __builtin_amdgcn_readfirstlane((int)b.y)}};
}
__device__ __forceinline__ Pages pages_at(const Listed& w, int step) {
    const Entries e = listed_at(w, step);
    return Pages{{e.id[0], e.id[1]}};
}
// (a list holds nothing but pages that are there)
__device__ __forceinline__ bool there(const Listed& w, int step, const Pages&, int u) { return step * 32 + 16 * u < w.end; }
__device__ __forceinline__ bool hole(const Listed& w, int step, const Pages&) { return step * 32 + 16 >= w.end; }
__device__ __forceinline__ Pages pages_for_mask(const Listed&, int) { return Pages{{0, 0}}; }
__device__ __forceinline__ Pages pages_by_number(const Listed& w, int step, const Pages&) { return pages_at(w, step); }
__device__ __forceinline__ Kept kept_at(const Listed& w, int step) {
    Kept r;
    if (w.keep) {
        const Entries e = listed_at(w, step);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = ((e.entry[u] << w.page_shift) + ((step * 32 + 16 * u) & (w.page - 1))) >> 2;
#pragma unroll
            for (int x = 0; x < 4; ++x) r.w[u][x] = w.keep[at + x];
        }
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int x = 0; x < 4; ++x) r.w[u][x] = 0x01010101u;
    }
    return r;
}
__device__ __forceinline__ bool left_out(const Listed& w, int t) {
    if (!w.keep) return false;
    const Entries e = listed_at(w, t >> 5);
    const int at = ((t & 16 ? e.entry[1] : e.entry[0]) << w.page_shift) + (t & (w.page - 1));
    return ((w.keep[at >> 2] >> (8 * (at & 3))) & 0xFF) == 0;
}

// The pages that any of several tokens has chosen; bit i: token i of them has.
struct Shared : Listed {
    uint32_t members;                                // in LDS
    uint32_t all;                                    // of the tokens
    int token;                                       // of the lane's row
};
struct Members { uint32_t m[2]; };
__device__ __forceinline__ Members members_at(const Shared& w, int step) {
    uint32_t a, b;
    asm volatile("ds_read_u16 %0, %2\n\tds_read_u16 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(a), "=&v"(b)
                 : "v"(w.members + 2 * min((step * 32) >> w.page_shift, w.last)), "v"(w.members + 2 * min((step * 32 + 16) >> w.page_shift, w.last)) : "memory");
    return Members{{(uint32_t)__builtin_amdgcn_readfirstlane((int)a), (uint32_t)__builtin_amdgcn_readfirstlane((int)b)}};
}
__device__ __forceinline__ bool uneven(const Shared& w, int step) {
    const Members m = members_at(w, step);
    return m.m[0] != w.all || m.m[1] != w.all;
}
__device__ __forceinline__ Sight sight_at(const Shared& w, int step) {
    const Members m = members_at(w, step);
    return Sight{{0u - ((m.m[0] >> w.token) & 1), 0u - ((m.m[1] >> w.token) & 1)}};
}

// tokens: that a block takes together; splits, most: parts of a list, and entries of a part
struct Chosen { const int32_t* list; int budget, splits, most, tokens; };
// Query rows of a part in the workspace: the heads that one unit has, sixteen at most.
__host__ __device__ __forceinline__ int part_rows(int G) { return G < 16 ? G : 16; }
constexpr int kChosenAt = (sizeof(AttendArgs) + 7) / 8 * 8;
constexpr int kChosenPartsAt = (kChosenAt + (int)sizeof(Chosen) + 7) / 8 * 8;

// What a block works on: 16 of the query heads of one token and K/V head and a part of its list; or all of those of several tokens.
struct Unit { int b, i, h, g0, split; };
__device__ __forceinline__ Unit unit_of(const AttendArgs& A, const Chosen& C, int x) {
    Unit u;
    u.split = x % C.splits; x /= C.splits;
    u.g0 = x % A.dim.tiles * 16; x /= A.dim.tiles;
    u.h = x % A.p.H; x /= A.p.H;
    const int groups = (A.dim.N + C.tokens - 1) / C.tokens;
    u.i = x % groups * C.tokens;
    u.b = x / groups;
    return u;
}
// The call as one of the tokens from i on looks to the others: their queries and outputs.
template <bool F32>
__device__ __forceinline__ void from_token(AttendArgs& A, int i) {
    const long q = (long)i * A.ql.token * (F32 ? 4 : 2), o = (long)i * A.ol.token * (F32 ? 4 : 2);
    A.q = static_cast<const char*>(A.q) + q;
    A.out = static_cast<char*>(A.out) + o;
    if (A.lse) A.lse += i;
}
// Entries that row i of a sample sees.
__device__ __forceinline__ int entries_seen(const Sample& s, int i) { return min(max(s.length - s.nq + i + 1, 0), s.length); }

// The entries of a token's list from v0 to v1 that count, by one wave: within the table, above all before them, and with something that
// the token sees.  each(entry, whether the lane's counts).  ahead: the first 64, which the caller has asked for.
__device__ __forceinline__ const int32_t* list_of(const AttendArgs& A, const Chosen& C, const Unit& u, int i) {
    return C.list + (((long)u.b * A.dim.N + i) * A.p.H + u.h) * C.budget;
}
template <class Each>
__device__ __forceinline__ void each_entry(const AttendArgs& A, const int32_t* from, int ahead, int seen, int v0, int v1, Each each) {
    const int lane = lane_id();
    const auto entry = [&](int v) {
        int e = ahead;
        if (v - lane != v0) e = from[min(v, v1 - 1)];
        return v < v1 && (uint32_t)e < (uint32_t)A.p.max_pages ? e : -1;
    };
    int before = -1;
    if (v0 > 0) {
        for (int v = lane; v < v0; v += kWave) before = max(before, entry(v));
        before = (int)~wave_min_u32(~(uint32_t)(before + 1)) - 1;
    }
    for (int base = v0; base < v1; base += kWave) {
        const int e = entry(base + lane);
        int top = e;                                 // the largest up to here
        const int after = __shfl_down(e, 1, kWave);
        if (__any(lane < kWave - 1 && base + lane < v1 - 1 && after <= e)) {                         // (a list that ascends is its own)
#pragma unroll
            for (int x = 1; x < kWave; x <<= 1) {
                const int other = __shfl_up(top, x, kWave);
                if (lane >= x) top = max(top, other);
            }
        }
        const int prior = __shfl_up(top, 1, kWave);
        const bool on = e > max(before, lane ? prior : -1) && ((long)e << A.p.page_shift) < seen;
        each(e, on);
        before = max(before, __builtin_amdgcn_readlane(top, kWave - 1));
    }
}

// A part of one token's list, by one wave: pages and entries.  Returns how many, and the tokens that they hold for it.
__device__ __forceinline__ int2 make_list(const AttendArgs& A, const int32_t* from, int ahead, const Unit& u, int seen, int v0, int v1, int2* list) {
    const int32_t* row = A.table + (long)u.b * A.p.max_pages;
    int n = 0, tokens = 0;
    each_entry(A, from, ahead, seen, v0, v1, [&](int e, bool on) {
        const int there = row[max(e, 0)], id = on ? c4_page_id(there, A.p.n_pages) : -1;
        const unsigned long long have = __ballot(id >= 0);
        if (id >= 0) list[n + lanes_below(have)] = int2{id, e};
        n += (int)__popcll(have);
        tokens += wave_sum_i(id >= 0 ? min(seen - (e << A.p.page_shift), A.p.page) : 0);
    });
    return int2{n, tokens};
}

// The lists of `n` tokens together, by all waves of the block.  s_any: 16 bits for each entry of the table.  Returns the number of pages.
__device__ __forceinline__ int make_shared_list(const AttendArgs& A, const Chosen& C, const Unit& u, const Sample& s, int n, uint32_t* s_any, int2* list,
                                                uint16_t* members, int* s_red) {
    const int tid = threadIdx.x, threads = blockDim.x, waves = threads >> 6;
    const int32_t* row = A.table + (long)u.b * A.p.max_pages;
    const int entries = c4_pages_of(entries_seen(s, u.i + n - 1), A.p.page_shift);
    for (int x = tid; x < (entries + 1) / 2; x += threads) s_any[x] = 0;
    block_sync_lds();
    for (int i = wave_id(); i < n; i += waves) {
        const int32_t* from = list_of(A, C, u, u.i + i);
        each_entry(A, from, from[min(lane_id(), C.budget - 1)], entries_seen(s, u.i + i), 0, C.budget, [&](int e, bool on) {
            if (on) atomicOr(&s_any[e >> 1], 1u << (16 * (e & 1) + i));
        });
    }
    block_sync_lds();
    int count = 0;
    for (int e0 = 0; e0 < entries; e0 += threads) {
        const int e = e0 + tid;
        const uint32_t m = e < entries ? (s_any[e >> 1] >> (16 * (e & 1))) & 0xFFFF : 0;
        const int id = m ? c4_page_id(row[e], A.p.n_pages) : -1;
        int total;
        const int at = block_rank(id >= 0, s_red, total);
        if (id >= 0) { list[count + at] = int2{id, e}; members[count + at] = (uint16_t)m; }
        count += total;
    }
    block_sync_lds();
    return count;
}

// A block per token, K/V head, 16 of its query heads and part of its list.
template <int D, bool F32, bool STREAM>
__global__ __launch_bounds__(F32 && D == 128 ? 256 : 512, F32 && D == 128 ? 3 : 4) void cache4_attend_chosen_kernel(AttendArgs A0, Chosen C0, Parts parts0)
{
    extern __shared__ f32x4 s_lds[];
    __shared__ int s_count[2];
    Sweep<D, F32, 1, STREAM> sw;
    Listed w;
    char* lds = reinterpret_cast<char*>(s_lds);
    {
        const AttendArgs A = argument<AttendArgs>(0);
        const Chosen C = argument<Chosen>(kChosenAt);
        const Unit u = unit_of(A, C, blockIdx.x);
        const int32_t* from = list_of(A, C, u, u.i);
        const int v0 = u.split * C.most, v1 = min(v0 + C.most, C.budget);
        int length = uniform(A.len)[u.b], nq = uniform(A.q_len ? A.q_len : A.len)[u.b], ahead = from[min(v0 + lane_id(), C.budget - 1)];
        asm volatile("" : "+s"(length), "+s"(nq), "+v"(ahead));      // (on their way together)
        Sample s{u.b, c4_clamp(length, 0, A.p.max_pages << A.p.page_shift), A.q_len ? c4_clamp(nq, 0, A.dim.N) : A.dim.N};
        if (u.i >= s.nq) return;
        int2* list = reinterpret_cast<int2*>(lds);   // (C.most entries; the rings and the join's sums are behind)
        AttendArgs T = A;
        from_token<F32>(T, u.i);
        sw.begin(T, Sample{u.b, 0, 1}, u.h, u.g0);   // (its queries are on their way while the list is made)
        if (wave_id() == 0) {
            const int2 made = make_list(A, from, ahead, u, entries_seen(s, u.i), v0, v1, list);
            if (lane_id() == 0) { s_count[0] = made.x; s_count[1] = made.y; }
        }
        __syncthreads();
        s.length = __builtin_amdgcn_readfirstlane(s_count[1]);
        s.nq = 1;
        sw.limit[0] = u.g0 + (lane_id() & 15) < A.dim.G ? s.length : 0;
        static_cast<Walk&>(w) = table_of(A, u.b);
        walk_of(w, A, s, u.h, 0, 0);
        w.list = lds_address(list);
        w.last = max(__builtin_amdgcn_readfirstlane(s_count[0]) - 1, 0);
        lds += (C.most + 1) / 2 * 16;
    }
    const Early early = early_pages(w, wave_id(), blockDim.x >> 6);
    sw.run(w, wave_id(), 0x7FFFFFFF, blockDim.x >> 6, lds + wave_id() * (sw.RING * sw.SLOT), early);
    __syncthreads();
    AttendArgs A = argument<AttendArgs>(0);
    const Chosen C = argument<Chosen>(kChosenAt);
    const Unit u = unit_of(A, C, blockIdx.x);
    from_token<F32>(A, u.i);
    const int rows = min(16, A.dim.G - u.g0);
    if (C.splits == 1) {
        join_waves<D, 1>(sw, rows, reinterpret_cast<float*>(lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
            store_out<D, F32>(A, u.b, u.h, u.g0 + row, part, x, m, l);
        });
    } else {
        const Parts parts = argument<Parts>(kChosenPartsAt);
        join_waves<D, 1>(sw, rows, reinterpret_cast<float*>(lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
            store_part<D>(parts, blockIdx.x, part_rows(A.dim.G), row, part, x, m, l);
        });
    }
}

// A block per K/V head and as many tokens as fill 16 query rows with their heads: over the pages that any of them has chosen, hidden from the
// others.  A key is converted once for all of them; tokens next to each other often choose the same pages.
template <int D, bool F32, bool STREAM>
__global__ __launch_bounds__(F32 && D == 128 ? 256 : 512, F32 && D == 128 ? 3 : 4) void cache4_attend_shared_kernel(AttendArgs A0, Chosen C0)
{
    extern __shared__ f32x4 s_lds[];
    __shared__ int s_red[8];
    Sweep<D, F32, 1, STREAM> sw;
    Shared w;
    char* lds = reinterpret_cast<char*>(s_lds);
    {
        AttendArgs A = argument<AttendArgs>(0);
        const Chosen C = argument<Chosen>(kChosenAt);
        const Unit u = unit_of(A, C, blockIdx.x);
        Sample s = sample_of(A, u.b);
        if (u.i >= s.nq) return;
        const int n = min(C.tokens, s.nq - u.i);
        int2* list = reinterpret_cast<int2*>(lds);   // (C.most entries, then which tokens have them; the rings and the join's sums are behind, and
                                                     // where those will be what make_shared_list goes by)
        uint16_t* members = reinterpret_cast<uint16_t*>(lds + (C.most + 1) / 2 * 16);
        lds += (C.most + 1) / 2 * 16 + (C.most + 7) / 8 * 16;
        AttendArgs T = A;
        from_token<F32>(T, u.i);
        sw.begin(T, Sample{u.b, 0, n}, u.h, 0);      // (its queries are on their way while the list is made)
        const int count = make_shared_list(A, C, u, s, n, reinterpret_cast<uint32_t*>(lds), list, members, s_red);
        // What a row sees ends within the list as it does in the sequence: in the last page that begins before.
        const int token = min((lane_id() & 15) / A.dim.G, n - 1), row_seen = entries_seen(s, u.i + token);
        int at = 0, limit = 0;                       // pages that begin before it
        for (int to = count; at < to;) {
            const int x = (at + to) >> 1;
            if ((list[x].y << A.p.page_shift) < row_seen) at = x + 1;
            else to = x;
        }
        if (at > 0) limit = ((at - 1) << A.p.page_shift) + min(row_seen - (list[at - 1].y << A.p.page_shift), A.p.page);
        static_cast<Walk&>(w) = table_of(A, u.b);
        s.length = __builtin_amdgcn_readlane(limit, (n - 1) * A.dim.G);
        s.nq = n;
        sw.limit[0] = (lane_id() & 15) < n * A.dim.G ? limit : 0;
        walk_of(w, A, s, u.h, 0, n * A.dim.G - 1);
        w.level = __builtin_amdgcn_readlane(limit, 0);                   // (the first token sees the least)
        w.list = lds_address(list);
        w.members = lds_address(members);
        w.all = (1u << n) - 1;
        w.token = token;
        w.last = max(count - 1, 0);
    }
    const Early early = early_pages(w, wave_id(), blockDim.x >> 6);
    sw.run(w, wave_id(), 0x7FFFFFFF, blockDim.x >> 6, lds + wave_id() * (sw.RING * sw.SLOT), early);
    __syncthreads();
    AttendArgs A = argument<AttendArgs>(0);
    const Chosen C = argument<Chosen>(kChosenAt);
    const Unit u = unit_of(A, C, blockIdx.x);
    const Sample s = sample_of(A, u.b);
    from_token<F32>(A, u.i);
    join_waves<D, 1>(sw, min(C.tokens, s.nq - u.i) * A.dim.G, reinterpret_cast<float*>(lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
        store_out<D, F32>(A, u.b, u.h, row, part, x, m, l);
    });
}

// Two sums of a row: (x, m, l) takes (y, my, ly) in.
template <int E>
__device__ __forceinline__ void join_sums(float (&x)[E], float& m, float& l, const float (&y)[E], float my, float ly) {
    const float top = fmaxf(m, my), a = fast_exp2(m - top), e = fast_exp2(my - top);
    m = top;
    l = l * a + ly * e;
#pragma unroll
    for (int z = 0; z < E; ++z) x[z] = fmaf(y[z], e, x[z] * a);
}

// The parts of a list: a block per token and query head, sixteen lanes per part, so that sixteen parts are on their way at once: what it waits
// for are its loads, one after another.  us for 64 heads of 25 parts 4.1 with the time of a launch, where a block with sixteen lanes per head took 10.1
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_attend_chosen_join_kernel(AttendArgs A, Chosen C, Parts parts)
{
    constexpr int E = D / 16;
    __shared__ float sums[4][16][E + 2];
    const int unit = blockIdx.x, row = blockIdx.y;
    const Chosen whole{C.list, C.budget, 1, C.budget, 1};
    const Unit u = unit_of(A, whole, unit);
    const Sample s = sample_of(A, u.b);
    const int wave = threadIdx.x >> 6, part = threadIdx.x & 15;
    if (u.i >= s.nq || u.g0 + row >= A.dim.G) return;          // (the whole block)
    float m = kNoKey, l = 0.f, acc[E] = {};
    for (int y = threadIdx.x >> 4; y < C.splits; y += 16) {
        const long at = ((long)unit * C.splits + y) * part_rows(A.dim.G) + row;
        const float2 ml = parts.ml[at];
        float v[E];
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
            const f32x4 w = reinterpret_cast<const f32x4*>(parts.o + at * D + part * E)[j];
#pragma unroll
            for (int z = 0; z < 4; ++z) v[4 * j + z] = w[z];
        }
        join_sums(acc, m, l, v, ml.x, ml.y);
    }
#pragma unroll
    for (int far = 16; far < 64; far *= 2) {
        float v[E];
#pragma unroll
        for (int z = 0; z < E; ++z) v[z] = __shfl_xor(acc[z], far);
        join_sums(acc, m, l, v, __shfl_xor(m, far), __shfl_xor(l, far));
    }
    if ((threadIdx.x & 48) == 0) {
#pragma unroll
        for (int z = 0; z < E; ++z) sums[wave][part][z] = acc[z];
        sums[wave][part][E] = m;
        sums[wave][part][E + 1] = l;
    }
    __syncthreads();
    if (threadIdx.x >= 16) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        float v[E];
#pragma unroll
        for (int z = 0; z < E; ++z) v[z] = sums[w][part][z];
        join_sums(acc, m, l, v, sums[w][part][E], sums[w][part][E + 1]);
    }
    from_token<F32>(A, u.i);
    store_out<D, F32>(A, u.b, u.h, u.g0 + row, part, acc, m, l);
}

// ------------------------------------------------------------------------------------------------ host

int bounds_impl(const void* cache, const int32_t* table, const int32_t* len, const int32_t* first, int8_t* bounds, uint8_t* scales,
                int B, int N, int H, int d, int n_pages, int page, int max_pages, void* stream)
{
    clear_error();
    Pool p;
    int rc = check_pool("cache4_bounds", H, d, n_pages, page, max_pages, &p);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N <= 0) return fail(MD_EINVAL, "cache4_bounds: sizes must be positive");
    if (!cache || !table || !len || !bounds || !scales) return fail(MD_EINVAL, "cache4_bounds: null pointer among the required arguments");
    if (!aligned16(cache) || !aligned16(bounds)) return fail(MD_EALIGN, "cache4_bounds: tensors must be 16-byte aligned");
    const int span = c4_span(N, page, max_pages);
    if ((long)B > (1l << 26) || (long)B * span * H > (1l << 25)) return fail(MD_ESHAPE, "cache4_bounds: %d samples of %d pages and %d heads are too many for one call", B, span, H);
    const size_t heads = (size_t)n_pages * H;
    const Range r[] = {{bounds, heads * 2 * d}, {scales, heads}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {first, first ? (size_t)B * 4 : 0}};
    rc = check_apart("cache4_bounds", r, 2, 6);
    if (rc != MD_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int units = B * span * H;
#define MD_C4_BOUNDS(D_, A_)                                                                                                              \
    MD_LAUNCH("cache4_bounds", st, (cache4_bounds_kernel<D_, A_>), (units + 3) / 4, 256, 0, static_cast<const uint8_t*>(cache), table, len, first, \
        bounds, scales, p, units, N, FastDiv::make(H), FastDiv::make(span))
    if (d == 128) { if (page >= 32) MD_C4_BOUNDS(128, 8); else MD_C4_BOUNDS(128, 4); }
    else if (page >= 64) MD_C4_BOUNDS(64, 8);
    else if (page >= 32) MD_C4_BOUNDS(64, 4);
    else MD_C4_BOUNDS(64, 2);
#undef MD_C4_BOUNDS
    return check_launch("cache4_bounds");
}

// Sizes of a call of the choice; scores follow in the workspace.
int choose_plan(const char* who, int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, Pool* p, Choose* A, size_t* bytes) {
    int rc = check_pool(who, H, d, n_pages, page, max_pages, p);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N <= 0 || Hq <= 0) return fail(MD_EINVAL, "%s: sizes must be positive", who);
    if (Hq % H || Hq > 65535) return fail(MD_ESHAPE, "%s: Hq=%d must be a multiple of H=%d", who, Hq, H);
    A->B = B; A->N = N; A->G = Hq / H; A->H = H; A->n_pages = n_pages; A->max_pages = max_pages; A->page_shift = p->page_shift;
    A->pitch = (max_pages + 15) / 16 * 16;
    A->lanes = 1;
    while (A->lanes < A->G && A->lanes < 16) A->lanes *= 2;
    A->subs = (A->G + 15) / 16;
    A->per = 16 / A->lanes;
    // (127 * 128 in each of 128 channels of 1024 heads are less than 2^31)
    if (A->G > 1024) return fail(MD_ESHAPE, "%s: %d query heads of one K/V head are too many", who, A->G);
    if ((long)N * A->G > (1l << 20)) return fail(MD_ESHAPE, "%s: %d tokens of %d query heads are too many for one call", who, N, Hq);
    if ((long)B * H > kMaxUnits || (long)B * H * N > kMaxUnits) return fail(MD_ESHAPE, "%s: %d samples of %d tokens and %d heads are too many for one call", who, B, N, H);
    // (blocks along y; and fewer than 2^23 scores are ranked at a time)
    if (max_pages > 65535 * 64 * kScoreTiles) return fail(MD_ESHAPE, "%s: %d pages are too many for one request", who, max_pages);
    A->tiles = (N + A->per - 1) / A->per;
    A->lds = 64 + 32 * (d + 16) + (size_t)(N < A->per ? N : A->per) * A->pitch * 4;
    A->together = A->subs == 1 && c4_choose_together((int64_t)B * H * A->tiles, A->pitch, A->lds);
    *bytes = A->together ? 256 : round_up((size_t)B * H * N * A->pitch * 4, 256);        // (scores of one launch for the next)
    return MD_OK;
}

int choose_impl(const void* q, int dtype, const int8_t* bounds, const uint8_t* scales, const int32_t* table, const int32_t* len, const int32_t* q_len,
                int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, int first_pages, int last_pages, int budget,
                int32_t* chosen, const md_kv_layout* q_layout, void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    const char* who = "cache4_choose";
    Pool p;
    Choose A{};
    size_t need = 0;
    int rc = choose_plan(who, B, N, Hq, H, d, n_pages, page, max_pages, &p, &A, &need);
    if (rc == MD_OK) rc = check_dtype(who, dtype);
    if (rc != MD_OK) return rc;
    if (budget <= 0 || first_pages < 0 || last_pages < 0) return fail(MD_EINVAL, "cache4_choose: budget must be positive, first_pages and last_pages not negative");
    if (budget > 1 << 26) return fail(MD_ESHAPE, "cache4_choose: a list of %d pages is too long", budget);        // (its places are counted in 31 bits, 1024 at a time)
    if ((long)first_pages + last_pages > budget) return fail(MD_EINVAL, "cache4_choose: %d first and %d last pages are more than the budget of %d", first_pages, last_pages, budget);
    if (!q || !bounds || !scales || !table || !len || !chosen) return fail(MD_EINVAL, "cache4_choose: null pointer among the required arguments");
    rc = read_layout(who, "q", q_layout, B, N, Hq, d, &A.ql);
    if (rc != MD_OK) return rc;
    if (!aligned16(q) || !aligned16(bounds)) return fail(MD_EALIGN, "cache4_choose: tensors must be 16-byte aligned");
    const size_t heads = (size_t)n_pages * H;
    const Range r[] = {{chosen, (size_t)B * N * H * budget * 4}, {workspace, workspace ? need : 0}, {q, rows_bytes(A.ql, B, N, Hq, d, dtype)}, {bounds, heads * 2 * d},
                       {scales, heads}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4}, {q_len, q_len ? (size_t)B * 4 : 0}};
    rc = check_apart(who, r, 2, 8);
    if (rc != MD_OK) return rc;
    if (!workspace || workspace_bytes < need)
        return fail(MD_EWORKSPACE, "cache4_choose: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(MD_EALIGN, "cache4_choose: workspace must be 256-byte aligned");
    A.q = q; A.bounds = bounds; A.scales = scales; A.table = table; A.len = len; A.q_len = q_len; A.chosen = chosen;
    A.scores = static_cast<float*>(workspace);
    A.first = first_pages; A.last = last_pages; A.budget = budget;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int tiles = A.tiles, chunks = (max_pages + 64 * kScoreTiles - 1) / (64 * kScoreTiles);
    const long blocks = (long)B * H * tiles;
    if (A.together) {
#define MD_C4_CHOOSE2(D_, F_, K_)                                                                                                         \
    MD_LAUNCH("cache4_score_choose", st, (cache4_score_choose_kernel<D_, F_, K_>), (int)blocks, 256, A.lds, A, FastDiv::make(tiles), FastDiv::make(H))
#define MD_C4_CHOOSE(D_, F_)                                                                                                              \
    do { if (max_pages <= 256) MD_C4_CHOOSE2(D_, F_, 4); else if (max_pages <= 768) MD_C4_CHOOSE2(D_, F_, 12); else MD_C4_CHOOSE2(D_, F_, 32); } while (0)
        if (d == 128) { if (dtype == MD_F32) MD_C4_CHOOSE(128, true); else MD_C4_CHOOSE(128, false); }
        else { if (dtype == MD_F32) MD_C4_CHOOSE(64, true); else MD_C4_CHOOSE(64, false); }
#undef MD_C4_CHOOSE
#undef MD_C4_CHOOSE2
        return check_launch(who);
    }
#define MD_C4_SCORE2(D_, F_, M_)                                                                                                          \
    MD_LAUNCH("cache4_score", st, (cache4_score_kernel<D_, F_, M_>), dim3((int)blocks, chunks), 256, 0, A, FastDiv::make(tiles), FastDiv::make(H))
#define MD_C4_SCORE(D_, F_) do { if (A.subs > 1) MD_C4_SCORE2(D_, F_, true); else MD_C4_SCORE2(D_, F_, false); } while (0)
    if (d == 128) { if (dtype == MD_F32) MD_C4_SCORE(128, true); else MD_C4_SCORE(128, false); }
    else { if (dtype == MD_F32) MD_C4_SCORE(64, true); else MD_C4_SCORE(64, false); }
#undef MD_C4_SCORE
#undef MD_C4_SCORE2
    // us for 8 lists of 2500 / 7500 scores: sixteen waves with eight each to a lane 6.3 / 7.4, by keys that are looked up again 6.6 / 11.6
    const int threads = max_pages <= 2048 ? 256 : 1024;
    const C4Lists l = c4_lists(B * H * N, threads);
    const dim3 lists(l.x, l.y);
    if (max_pages <= 2048) MD_LAUNCH("cache4_choose", st, (cache4_choose_block_kernel<4>), lists, threads, 0, A, FastDiv::make(N), FastDiv::make(H));
    else if (max_pages <= 8192) MD_LAUNCH("cache4_choose", st, (cache4_choose_block_kernel<16>), lists, threads, 0, A, FastDiv::make(N), FastDiv::make(H));
    else MD_LAUNCH("cache4_choose", st, (cache4_choose_kernel), lists, threads, 0, A, FastDiv::make(N), FastDiv::make(H));
    return check_launch(who);
}

struct ChosenPlan {
    C4Chosen cut;
    Parts parts;
    int tiles;
    long units;
    size_t lds, bytes;
};
// max_pages: of the block table, or 0 where only the workspace's size is asked for
ChosenPlan chosen_plan(void* workspace, bool f32, int B, int N, int Hq, int d, int budget, int max_pages, const Pool& p) {
    ChosenPlan a;
    const int G = Hq / p.H;
    a.tiles = (G + 15) / 16;
    a.cut = c4_chosen(f32, d, B, N, G, p.H, budget, p.page, max_pages);
    a.units = (long)B * ((N + a.cut.tokens - 1) / a.cut.tokens) * p.H * a.tiles;
    const int rows = a.cut.tokens * G < 16 ? a.cut.tokens * G : 16;
    const size_t join = sizeof(float) * ((size_t)a.cut.waves * rows * (d + 4) + 2 * a.cut.waves * 16), ring = (size_t)a.cut.waves * kRing * (32 * d + 256);
    const size_t list = (size_t)(a.cut.most + 1) / 2 * 16 + (a.cut.tokens > 1 ? (size_t)(a.cut.most + 7) / 8 * 16 : 0);
    a.lds = list + (join > ring ? join : ring);      // (the ring is more than two bytes for each entry of a table that lists are shared in)
    // (parts of lists are joined through the workspace.  Tokens that go together have none; without max_pages nobody goes together: the most that
    // a call may need)
    const size_t places = a.cut.splits > 1 ? (size_t)a.units * a.cut.splits * part_rows(G) : 0;
    Carver c(workspace);
    a.parts.o = c.take<float>(places * d);
    a.parts.ml = c.take<float2>(places);
    a.parts.blocks = a.parts.least = 0;
    a.bytes = c.off > 256 ? c.off : 256;
    return a;
}
int check_chosen(const char* who, int B, int N, int Hq, int H, int budget) {
    if (B <= 0 || N <= 0 || Hq <= 0 || budget <= 0) return fail(MD_EINVAL, "%s: sizes must be positive", who);
    if (Hq % H || Hq > 65535) return fail(MD_ESHAPE, "%s: Hq=%d must be a multiple of H=%d", who, Hq, H);
    if (budget > (1 << 26) || (double)B * N * H * ((Hq / H + 15) / 16) * ((budget + kC4ListMost - 1) / kC4ListMost) > (double)kMaxUnits)
        return fail(MD_ESHAPE, "%s: %d samples of %d tokens and %d heads over %d pages are too many for one call", who, B, N, Hq, budget);
    return MD_OK;
}

size_t attend_chosen_bytes(int B, int N, int Hq, int H, int d, int budget, int page) {
    Pool p;
    if (check_pool("cache4_attend_chosen", H, d, 1, page, 1, &p) != MD_OK || check_chosen("cache4_attend_chosen", B, N, Hq, H, budget) != MD_OK) return 0;
    const size_t x = chosen_plan(nullptr, false, B, N, Hq, d, budget, 0, p).bytes, y = chosen_plan(nullptr, true, B, N, Hq, d, budget, 0, p).bytes;
    return x > y ? x : y;
}

int attend_chosen_impl(const void* q, int dtype, const void* cache, const int32_t* table, const int32_t* len, const int32_t* q_len, const uint8_t* keep,
                       const int32_t* chosen, int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, int budget, float softmax_scale,
                       void* out, float* lse, const md_kv_layout* q_layout, const md_kv_layout* out_layout,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    const char* who = "cache4_attend_chosen";
    Pool p;
    int rc = check_pool(who, H, d, n_pages, page, max_pages, &p);
    if (rc == MD_OK) rc = check_dtype(who, dtype);
    if (rc == MD_OK) rc = check_chosen(who, B, N, Hq, H, budget);
    if (rc != MD_OK) return rc;
    if (!q || !cache || !table || !len || !chosen || !out) return fail(MD_EINVAL, "cache4_attend_chosen: null pointer among the required arguments");
    if (!(softmax_scale > 0.f) || std::isinf(softmax_scale * kLog2eC))
        return fail(MD_EINVAL, "cache4_attend_chosen: softmax_scale must be positive and finite, times log2(e) too");
    KvLayout ql, ol;
    rc = read_layout(who, "q", q_layout, B, N, Hq, d, &ql);
    if (rc == MD_OK) rc = read_layout(who, "out", out_layout, B, N, Hq, d, &ol);
    if (rc != MD_OK) return rc;
    if (!aligned16(q) || !aligned16(out) || !aligned16(cache) || (reinterpret_cast<uintptr_t>(keep) & 3u))
        return fail(MD_EALIGN, "cache4_attend_chosen: tensors must be 16-byte aligned, keep 4-byte aligned");
    const ChosenPlan plan = chosen_plan(workspace, dtype == MD_F32, B, N, Hq, d, budget, max_pages, p);
    const size_t need = plan.bytes;
    const Range r[] = {{out, rows_bytes(ol, B, N, Hq, d, dtype)}, {lse, lse ? (size_t)B * Hq * N * 4 : 0}, {workspace, workspace ? need : 0},
                       {q, rows_bytes(ql, B, N, Hq, d, dtype)}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {q_len, q_len ? (size_t)B * 4 : 0}, {keep, keep ? (size_t)B * max_pages * page : 0}, {chosen, (size_t)B * N * H * budget * 4}};
    rc = check_apart(who, r, 3, 10);
    if (rc != MD_OK) return rc;
    if (!workspace || workspace_bytes < need)
        return fail(MD_EWORKSPACE, "cache4_attend_chosen: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(MD_EALIGN, "cache4_attend_chosen: workspace must be 256-byte aligned");
    const AttendArgs A{q, static_cast<const uint8_t*>(cache), table, len, q_len, keep, out, lse, p, AttendDims{B, N, Hq / H, plan.tiles}, softmax_scale, ql, ol};
    const Chosen C{chosen, budget, plan.cut.splits, plan.cut.most, plan.cut.tokens};
    const int blocks = (int)(plan.units * plan.cut.splits);
    const bool stream_once = pool_bytes(p) > (size_t)128 << 20;
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_CHOSEN(D_, F_, S_)                                                                                                          \
    do {                                                                                                                                  \
        if (C.tokens > 1) { MD_LAUNCH("cache4_attend_shared", st, (cache4_attend_shared_kernel<D_, F_, S_>), blocks, plan.cut.waves * 64, plan.lds, A, C); break; } \
        MD_LAUNCH("cache4_attend_chosen", st, (cache4_attend_chosen_kernel<D_, F_, S_>), blocks, plan.cut.waves * 64, plan.lds, A, C, plan.parts); \
        if (C.splits > 1) MD_LAUNCH("cache4_chosen_join", st, (cache4_attend_chosen_join_kernel<D_, F_>), dim3((unsigned)plan.units, (unsigned)part_rows(A.dim.G)), 256, 0, A, C, plan.parts); \
    } while (0)
#define MD_C4_CHOSEN_S(D_, F_) do { if (stream_once) MD_C4_CHOSEN(D_, F_, true); else MD_C4_CHOSEN(D_, F_, false); } while (0)
    if (d == 128) { if (dtype == MD_F32) MD_C4_CHOSEN_S(128, true); else MD_C4_CHOSEN_S(128, false); }
    else { if (dtype == MD_F32) MD_C4_CHOSEN_S(64, true); else MD_C4_CHOSEN_S(64, false); }
#undef MD_C4_CHOSEN_S
#undef MD_C4_CHOSEN
    return check_launch(who);
}

}  // namespace
}  // namespace md

extern "C" int mustdrop_cache4_bounds(
    const void* cache, const int32_t* table, const int32_t* len, const int32_t* first, int8_t* bounds, uint8_t* scales,
    int B, int N, int H, int d, int n_pages, int page, int max_pages, void* stream)
{
    return md::bounds_impl(cache, table, len, first, bounds, scales, B, N, H, d, n_pages, page, max_pages, stream);
}

extern "C" size_t mustdrop_cache4_choose_workspace_bytes(int B, int N, int Hq, int H, int d, int max_pages, int page)
{
    md::clear_error();
    md::Pool p;
    md::Choose A{};
    size_t bytes = 0;
    return md::choose_plan("cache4_choose", B, N, Hq, H, d, 1, page, max_pages, &p, &A, &bytes) == MD_OK ? bytes : 0;
}

extern "C" int mustdrop_cache4_choose(
    const void* q, md_dtype dtype, const int8_t* bounds, const uint8_t* scales, const int32_t* table, const int32_t* len, const int32_t* q_len,
    int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, int first_pages, int last_pages, int budget,
    int32_t* chosen, const md_kv_layout* q_layout, void* workspace, size_t workspace_bytes, void* stream)
{
    return md::choose_impl(q, dtype, bounds, scales, table, len, q_len, B, N, Hq, H, d, n_pages, page, max_pages, first_pages, last_pages, budget,
                           chosen, q_layout, workspace, workspace_bytes, stream);
}

extern "C" size_t mustdrop_cache4_attend_chosen_workspace_bytes(int B, int N, int Hq, int H, int d, int budget, int page)
{
    md::clear_error();
    return md::attend_chosen_bytes(B, N, Hq, H, d, budget, page);
}

extern "C" int mustdrop_cache4_attend_chosen(
    const void* q, md_dtype dtype, const void* cache, const int32_t* table, const int32_t* len, const int32_t* q_len, const uint8_t* keep,
    const int32_t* chosen, int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, int budget, float softmax_scale,
    void* out, float* lse, const md_kv_layout* q_layout, const md_kv_layout* out_layout,
    void* workspace, size_t workspace_bytes, void* stream)
{
    return md::attend_chosen_impl(q, dtype, cache, table, len, q_len, keep, chosen, B, N, Hq, H, d, n_pages, page, max_pages, budget, softmax_scale,
                                  out, lse, q_layout, out_layout, workspace, workspace_bytes, stream);
}
