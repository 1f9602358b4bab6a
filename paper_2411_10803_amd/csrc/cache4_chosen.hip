// Attention over a part of the cache held in 4 bits.
//
//   cache4_bounds_kernel          each page's largest and smallest key values, channel by channel, in 8 bits
//   cache4_score_kernel           bounds and queries -> a score for each token, K/V head and page
//   cache4_choose_kernel          scores -> the pages to read
//   cache4_attend_chosen_kernel   softmax(scale Q K^T) V over them
//   cache4_attend_chosen_join_kernel   the same where a list is cut into parts
//
// The score of a page is the sum over the G query heads of max over [smallest, largest] of q . k, which is no less than the sum of any of its
// keys' own scores: max(q a, q b) = max(q, 0) a + min(q, 0) b for a >= b, so that it is one matrix product with twice the channels.
// Bounds and queries are whole numbers of 8 bits times a power of two: their sums are exact, whatever the order, and so is the choice.
#include "cache4_host.hpp"

namespace md {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------------ bounds

// Maxima over lanes that differ in bit S, of 2 S numbers: lanes with the bit set go on with the upper S, the others with the lower.
template <int S>
__device__ __forceinline__ void halve(float (&v)[64], int lane) {
#pragma unroll
    for (int c = 0; c < S; ++c) {
        const bool up = lane & S;
        const float keep = up ? v[c + S] : v[c], give = up ? v[c] : v[c + S];
        v[c] = fmaxf(keep, __shfl_xor(give, S, kWave));
    }
}

// A wave per page and head.  A lane loads 16 bytes, 32 channels of one scale, of every 16th (d = 64: 32nd) token, and keeps the largest
// of their values and of the values with their signs turned: 64 numbers.  The lanes of one group then halve these among them, until each
// has 4 (2) channels of the one kind, which is a word (half of one) of the result.
template <int D>
__global__ __launch_bounds__(256) void cache4_bounds_kernel(
    const uint8_t* __restrict__ cache, const int32_t* __restrict__ table, const int32_t* __restrict__ len, const int32_t* __restrict__ first,
    int8_t* __restrict__ bounds, uint8_t* __restrict__ scales, Pool p, int units, int N, FastDiv heads, FastDiv span)
{
    constexpr int GROUPS = D / 32, TOKENS = kWave / GROUPS;
    const int unit = (int)blockIdx.x * 4 + wave_id(), lane = lane_id();
    if (unit >= units) return;
    const int bx = heads.div(unit), h = unit - bx * heads.d, b = span.div(bx), x = bx - b * span.d;
    const int length = c4_clamp(len[b], 0, p.max_pages << p.page_shift), from = first ? max(first[b], 0) : 0;
    const long e = (long)(from >> p.page_shift) + x;
    if ((e << p.page_shift) >= min((long)from + N, (long)length)) return;
    const int id = c4_page_id(table[(long)b * p.max_pages + e], p.n_pages);
    if (id < 0) return;
    const int live = min(length - (int)(e << p.page_shift), p.page);
    const uint8_t* base = cache + ((long)id * p.H + h) * p.stride;
    const int group = lane & (GROUPS - 1), t0 = lane / GROUPS;
    float v[64];                                     // largest, then largest of the negative, of 32 channels
#pragma unroll
    for (int c = 0; c < 64; ++c) v[c] = -INFINITY;
    bool bad = false;
    for (int t = t0; t < live; t += TOKENS) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(base + c4_k_codes(t, D) + group * 16);
        const uint32_t code = base[c4_k_scales(p.page, t, D) + group];
        const float s = scale_of(code);
        bad |= code >= 253;                          // (6 * 2^126 is no number of fp32)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], s, 1),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], s, 3)};
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float f = y[c >> 1][c & 1];
                v[j * 8 + c] = fmaxf(v[j * 8 + c], f);
                v[32 + j * 8 + c] = fmaxf(v[32 + j * 8 + c], -f);
            }
        }
    }
    halve<32>(v, lane);
    halve<16>(v, lane);
    halve<8>(v, lane);
    halve<4>(v, lane);
    if (D == 64) halve<2>(v, lane);
    constexpr int LEFT = D == 128 ? 4 : 2;
    float most = v[0];
#pragma unroll
    for (int c = 1; c < LEFT; ++c) most = fmaxf(most, v[c]);
    most = wave_max(most);                           // the largest magnitude: of a channel's largest and smallest value one has it
    const bool none = __any(bad);
    const int ex = most > 0.f ? max((int)(__float_as_uint(most) >> 23) - 127 - 6, -126) : -126;
    const bool least = lane & 32;
    uint32_t word = 0;
#pragma unroll
    for (int c = 0; c < LEFT; ++c) {
        const int up = none ? 0 : (int)ceilf(__builtin_amdgcn_ldexpf(v[c], -ex));
        word |= (uint32_t)((least ? -up : up) & 0xFF) << (8 * c);
    }
    const int channel = group * 32 + (lane & 16) + (lane & 8) + (lane & 4) + (D == 64 ? (lane & 2) : 0);
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
    int lanes, subs, per;                            // query heads of a token side by side (a power of two), tiles of them, tokens of a tile
};

// Pages that row i of sample b sees; -1 where there is no such row.
__device__ __forceinline__ int pages_seen(const Choose& A, int b, int i) {
    const int length = c4_clamp(A.len[b], 0, A.max_pages << A.page_shift), nq = A.q_len ? c4_clamp(A.q_len[b], 0, A.N) : A.N;
    if (i >= nq) return -1;
    return c4_pages_of(min(max(length - nq + i + 1, 0), length), A.page_shift);
}

// The whole numbers of a lane's 16 channels of one query, as bytes: those above 0, and those below.
__device__ __forceinline__ void whole_bytes(const float (&x)[16], int shift, bool ok, i32x4& above, i32x4& below) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t a = 0, b = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = ok ? c4_clamp((int)rintf(__builtin_amdgcn_ldexpf(x[4 * w + j], shift)), -127, 127) : 0;
            a |= (uint32_t)max(n, 0) << (8 * j);
            b |= (uint32_t)(min(n, 0) & 0xFF) << (8 * j);
        }
        above[w] = (int)a;
        below[w] = (int)b;
    }
}

template <bool F32>
__device__ __forceinline__ void load_16(const void* base, long at, float (&x)[16]) {
    if (F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + at + 4 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at + 8 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[8 * i + 2 * j] = bf16_lo(v[j]); x[8 * i + 2 * j + 1] = bf16_hi(v[j]); }
        }
    }
}

// A wave: 16 query rows (the G heads of some tokens, filled up with zeros to a power of two) against TILES tiles of 16 pages.  Lane (n, lb)
// has bytes lb * 16 .. + 15 of every 64 of row n of either operand.
constexpr int kScoreTiles = 4;
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_score_kernel(Choose A, FastDiv tiles, FastDiv heads)
{
    constexpr int Y = D / 64;
    const int lane = lane_id(), n = lane & 15, lb = lane >> 4;
    const int bh = tiles.div(blockIdx.x), tile = blockIdx.x - bh * tiles.d, b = heads.div(bh), h = bh - b * heads.d;
    const int nq = A.q_len ? c4_clamp(A.q_len[b], 0, A.N) : A.N;
    const int i = tile * A.per + n / A.lanes, g0 = n & (A.lanes - 1), last = min(nq, (tile + 1) * A.per) - 1;
    if (tile * A.per >= nq) return;
    const int seen = pages_seen(A, b, last), first = ((int)blockIdx.y * 4 + wave_id()) * kScoreTiles;
    if (first * 16 >= seen) return;
    // the largest magnitude of a token's queries
    uint32_t most = 0;
    for (int s = 0; s < A.subs; ++s) {
        const int g = s * 16 + g0;
        if (i >= nq || g >= A.G) continue;
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            float x[16];
            load_16<F32>(A.q, (long)b * A.ql.batch + (long)i * A.ql.token + (long)(h * A.G + g) * A.ql.head + y * 64 + lb * 16, x);
#pragma unroll
            for (int j = 0; j < 16; ++j) most = max(most, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        }
    }
    most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32, kWave));
    for (int x = 1; x < A.lanes; x <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, x, kWave));
    const bool ok = most > 0 && most < 0x7F800000u;
    const int shift = 7 - __builtin_amdgcn_frexp_expf(__uint_as_float(most));
    i32x4 acc[kScoreTiles] = {};
    int code[kScoreTiles];                           // of the lane's page n in each tile: its scale; 256: no page
#pragma unroll
    for (int t = 0; t < kScoreTiles; ++t) code[t] = 256;
    for (int s = 0; s < A.subs; ++s) {
        const int g = s * 16 + g0;
        i32x4 above[Y], below[Y];
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            float x[16] = {};
            if (i < nq && g < A.G) load_16<F32>(A.q, (long)b * A.ql.batch + (long)i * A.ql.token + (long)(h * A.G + g) * A.ql.head + y * 64 + lb * 16, x);
            whole_bytes(x, shift, ok, above[y], below[y]);
        }
#pragma unroll
        for (int t = 0; t < kScoreTiles; ++t) {
            const int e = (first + t) * 16 + n;
            i32x4 hi[Y] = {}, lo[Y] = {};
            if (e < seen) {
                const int id = c4_page_id(A.table[(long)b * A.max_pages + e], A.n_pages);
                if (id >= 0) {
                    const long at = (long)id * A.H + h;
                    code[t] = A.scales[at];
                    const int8_t* from = A.bounds + at * (2 * D) + lb * 16;
#pragma unroll
                    for (int y = 0; y < Y; ++y) {
                        hi[y] = *reinterpret_cast<const i32x4*>(from + y * 64);
                        lo[y] = *reinterpret_cast<const i32x4*>(from + D + y * 64);
                    }
                }
            }
#pragma unroll
            for (int y = 0; y < Y; ++y) {
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi[y], above[y], acc[t], 0, 0, 0);
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(lo[y], below[y], acc[t], 0, 0, 0);
            }
        }
    }
    float* to = A.scores + ((long)bh * A.N + i) * A.pitch;
#pragma unroll
    for (int t = 0; t < kScoreTiles; ++t) {
        const int e0 = (first + t) * 16 + 4 * lb;    // acc[t][x]: page e0 + x, query n
        f32x4 score;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            int sum = acc[t][x];
            for (int m = 1; m < A.lanes; m <<= 1) sum += __shfl_xor(sum, m, kWave);
            const int c = __shfl(code[t], 4 * lb + x, kWave);
            score[x] = c == 256 ? -INFINITY : c == 255 ? INFINITY : __builtin_amdgcn_ldexpf((float)sum, c - 127);
        }
        if (i < nq && g0 == 0 && e0 < seen) *reinterpret_cast<f32x4*>(to + e0) = score;
    }
}

// ------------------------------------------------------------------------------------------------ choice

// Larger scores first, of equal ones the first page; never 0.
__device__ __forceinline__ uint64_t page_key(float score, int e) {
    const uint32_t u = __float_as_uint(score + 0.f), up = u & 0x80000000u ? ~u : u | 0x80000000u;       // (-0 is 0)
    return ((uint64_t)up << 32) | (uint32_t)(0x7FFFFFFF - e);
}

// A block per token and K/V head.
__global__ __launch_bounds__(256) void cache4_choose_kernel(Choose A, FastDiv tokens, FastDiv heads)
{
    __shared__ int s_hist[kSelectHistInts], s_red[4];
    const int bh = tokens.div(blockIdx.x), i = blockIdx.x - bh * tokens.d, b = heads.div(bh), h = bh - b * heads.d;
    const int P = pages_seen(A, b, i);
    if (P < 0) return;
    const float* score = A.scores + (long)blockIdx.x * A.pitch;
    int32_t* to = A.chosen + (((long)b * A.N + i) * A.H + h) * A.budget;
    const int lo = min(A.first, P), hi = max(P - A.last, lo), always = lo + P - hi;      // pages lo .. hi - 1 are ranked
    int taken = P;
    SelectBound bound{0, 63};
    if (P > A.budget) {
        for (int x = threadIdx.x; x < kSelectHistInts; x += 256) s_hist[x] = 0;
        __syncthreads();
        bound = block_select_keys([&](auto f) {
            for (int e = lo + (int)threadIdx.x; e < hi; e += 256) f(page_key(score[e], e));
        }, A.budget - always, s_hist);
        taken = A.budget;
    }
    int done = 0;
    for (int e0 = 0; e0 < P; e0 += 256) {
        const int e = e0 + threadIdx.x;
        bool in = e < P;
        if (in && P > A.budget && e >= lo && e < hi) in = A.budget > always && (page_key(score[e], e) >> bound.shift) >= bound.bound;
        int total;
        const int at = block_rank(in, s_red, total);
        if (in && done + at < A.budget) to[done + at] = e;
        done += total;
    }
    for (int x = taken + threadIdx.x; x < A.budget; x += 256) to[x] = -1;
}

// ------------------------------------------------------------------------------------------------ attention

// A walk over the pages of a list, which lies in LDS: page numbers and entries of the block table.  Positions of the walk count the
// list's tokens, one page after the other.
struct Listed : Walk {
    const int2* list;
    int last;                                        // of the list
};
__device__ __forceinline__ int2 listed_at(const Listed& w, int t) {
    const int2 v = w.list[min(t >> w.page_shift, w.last)];
    return int2{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y)};
}
__device__ __forceinline__ Pages pages_at(const Listed& w, int step) {
    Pages r;
#pragma unroll
    for (int u = 0; u < 2; ++u) r.id[u] = listed_at(w, step * 32 + 16 * u).x;
    return r;
}
__device__ __forceinline__ int entry_of(const Listed& w, int t) { return (listed_at(w, t).y << w.page_shift) + (t & (w.page - 1)); }
__device__ __forceinline__ Kept kept_at(const Listed& w, int step) {
    Kept r;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (w.keep) {
            const int at = entry_of(w, step * 32 + 16 * u) >> 2;
#pragma unroll
            for (int x = 0; x < 4; ++x) r.w[u][x] = w.keep[at + x];
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x) r.w[u][x] = 0x01010101u;
        }
    }
    return r;
}
__device__ __forceinline__ bool left_out(const Listed& w, int t) {
    if (!w.keep) return false;
    const int at = entry_of(w, t);
    return ((w.keep[at >> 2] >> (8 * (at & 3))) & 0xFF) == 0;
}

struct Chosen { const int32_t* list; int budget, splits, most; };
constexpr int kChosenAt = (sizeof(AttendArgs) + 7) / 8 * 8;

// What a block works on: a part of the list of one token and K/V head, and 16 of its query heads.
struct Unit { int b, i, h, g0, split; };
__device__ __forceinline__ Unit unit_of(const AttendArgs& A, const Chosen& C) {
    Unit u;
    int x = blockIdx.x;
    u.split = x % C.splits; x /= C.splits;
    u.g0 = x % A.dim.tiles * 16; x /= A.dim.tiles;
    u.h = x % A.p.H; x /= A.p.H;
    u.i = x % A.dim.N;
    u.b = x / A.dim.N;
    return u;
}
// The call as one of a single token looks to the others: that token's query and outputs.
template <bool F32>
__device__ __forceinline__ void only_token(AttendArgs& A, int i) {
    const long q = (long)i * A.ql.token * (F32 ? 4 : 2), o = (long)i * A.ol.token * (F32 ? 4 : 2);
    A.q = static_cast<const char*>(A.q) + q;
    A.out = static_cast<char*>(A.out) + o;
    if (A.lse) A.lse += i;
}

// The entries of a part that count, in order, by the block's first wave: within the table, above all before them, with something that
// the token sees, and with a page.  Returns the tokens that they hold for it.
__device__ __forceinline__ int make_list(const AttendArgs& A, const Chosen& C, const Unit& u, int seen, int2* list, int& count) {
    const int lane = lane_id();
    const int32_t* from = C.list + (((long)u.b * A.dim.N + u.i) * A.p.H + u.h) * C.budget;
    const int32_t* row = A.table + (long)u.b * A.p.max_pages;
    const int v0 = u.split * C.most, v1 = min(v0 + C.most, C.budget);
    const auto entry = [&](int v) {
        const int e = v < v1 ? from[v] : -1;
        return (uint32_t)e < (uint32_t)A.p.max_pages ? e : -1;
    };
    int before = -1;
    for (int v = lane; v < v0; v += kWave) before = max(before, entry(v));
    before = (int)~wave_min_u32(~(uint32_t)(before + 1)) - 1;
    int n = 0, tokens = 0;
    for (int base = v0; base < v1; base += kWave) {
        const int e = entry(base + lane);
        int top = e;                                 // the largest up to here
#pragma unroll
        for (int x = 1; x < kWave; x <<= 1) {
            const int other = __shfl_up(top, x, kWave);
            if (lane >= x) top = max(top, other);
        }
        const int prior = __shfl_up(top, 1, kWave);
        const bool rises = e >= 0 && e > max(before, lane ? prior : -1);
        int id = -1;
        if (rises && ((long)e << A.p.page_shift) < seen) id = c4_page_id(row[e], A.p.n_pages);
        const unsigned long long on = __ballot(id >= 0);
        if (id >= 0) list[n + lanes_below(on)] = int2{id, e};
        n += __popcll(on);
        int mine = id >= 0 ? min(seen - (e << A.p.page_shift), A.p.page) : 0;
        tokens += wave_sum_i(mine);
        before = max(before, __builtin_amdgcn_readlane(top, kWave - 1));
    }
    count = n;
    return tokens;
}

template <int D, bool F32, bool STREAM>
__global__ __launch_bounds__(F32 && D == 128 ? 256 : 512, F32 && D == 128 ? 3 : 4) void cache4_attend_chosen_kernel(AttendArgs A0, Chosen C0, Parts parts0)
{
    extern __shared__ f32x4 s_lds[];
    __shared__ int s_count[2];
    Sweep<D, F32, 1, STREAM> sw;
    Listed w;
    char* lds = reinterpret_cast<char*>(s_lds);
    int2* list = reinterpret_cast<int2*>(lds);       // (C.most entries; the rings and the join's sums are behind)
    {
        AttendArgs A = argument<AttendArgs>(0);
        const Chosen C = argument<Chosen>(kChosenAt);
        const Unit u = unit_of(A, C);
        Sample s = sample_of(A, u.b);
        if (u.i >= s.nq) return;
        const int seen = min(max(s.length - s.nq + u.i + 1, 0), s.length);
        if (wave_id() == 0) {
            int count;
            const int tokens = make_list(A, C, u, seen, list, count);
            if (lane_id() == 0) { s_count[0] = count; s_count[1] = tokens; }
        }
        __syncthreads();
        s.length = __builtin_amdgcn_readfirstlane(s_count[1]);
        s.nq = 1;
        static_cast<Walk&>(w) = table_of(A, u.b);
        only_token<F32>(A, u.i);
        // 16 query heads from g0 on, as rows of a K/V head
        sw.begin(A, s, u.h, u.g0);
        walk_of(w, A, s, u.h, 0, 0);
        w.list = list;
        w.last = max(__builtin_amdgcn_readfirstlane(s_count[0]) - 1, 0);
        lds += (C.most + 1) / 2 * 16;
    }
    const Early early = early_pages(w, wave_id(), blockDim.x >> 6);
    sw.run(w, wave_id(), 0x7FFFFFFF, blockDim.x >> 6, lds + wave_id() * (sw.RING * sw.SLOT), early);
    __syncthreads();
    AttendArgs A = argument<AttendArgs>(0);
    const Chosen C = argument<Chosen>(kChosenAt);
    const Unit u = unit_of(A, C);
    only_token<F32>(A, u.i);
    const int rows = min(16, A.dim.G - u.g0);
    if (C.splits == 1) {
        join_waves<D, 1>(sw, rows, reinterpret_cast<float*>(lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
            store_out<D, F32>(A, u.b, u.h, u.g0 + row, part, x, m, l);
        });
    } else {
        const Parts parts = argument<Parts>((kChosenAt + (int)sizeof(Chosen) + 7) / 8 * 8);
        join_waves<D, 1>(sw, rows, reinterpret_cast<float*>(lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
            store_part<D>(parts, blockIdx.x, 16, row, part, x, m, l);
        });
    }
}

// The parts of a list: a block per token, K/V head and 16 query heads, sixteen lanes per head.
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_attend_chosen_join_kernel(AttendArgs A, Chosen C, Parts parts)
{
    const int unit = blockIdx.x;
    const Chosen whole{C.list, C.budget, 1, C.budget};
    const Unit u = unit_of(A, whole);
    const Sample s = sample_of(A, u.b);
    const int row = threadIdx.x >> 4, part = threadIdx.x & 15;
    if (u.i >= s.nq || u.g0 + row >= A.dim.G) return;
    float m = kNoKey, l = 0.f, acc[D / 16] = {};
    for (int y = 0; y < C.splits; ++y) {
        const long at = ((long)unit * C.splits + y) * 16 + row;
        const float2 ml = parts.ml[at];
        const float top = fmaxf(m, ml.x), a = fast_exp2(m - top), e = fast_exp2(ml.x - top);
        m = top;
        l = l * a + ml.y * e;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const f32x4 v = reinterpret_cast<const f32x4*>(parts.o + at * D + part * (D / 16))[j];
#pragma unroll
            for (int z = 0; z < 4; ++z) acc[4 * j + z] = fmaf(v[z], e, acc[4 * j + z] * a);
        }
    }
    only_token<F32>(A, u.i);
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
#define MD_C4_BOUNDS(D_)                                                                                                                  \
    MD_LAUNCH("cache4_bounds", st, (cache4_bounds_kernel<D_>), (units + 3) / 4, 256, 0, static_cast<const uint8_t*>(cache), table, len, first, \
        bounds, scales, p, units, N, FastDiv::make(H), FastDiv::make(span))
    if (d == 128) MD_C4_BOUNDS(128); else MD_C4_BOUNDS(64);
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
    if ((long)N * A->G > (1l << 20)) return fail(MD_ESHAPE, "%s: %d tokens of %d query heads are too many for one call", who, N, Hq);
    if ((long)B * H > kMaxUnits || (long)B * H * N > kMaxUnits) return fail(MD_ESHAPE, "%s: %d samples of %d tokens and %d heads are too many for one call", who, B, N, H);
    *bytes = round_up((size_t)B * H * N * A->pitch * 4, 256);
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
    const int tiles = (N + A.per - 1) / A.per, chunks = (max_pages + 64 * kScoreTiles - 1) / (64 * kScoreTiles);
    if (chunks > 65535) return fail(MD_ESHAPE, "cache4_choose: %d pages are too many for one request", max_pages);
#define MD_C4_SCORE(D_, F_)                                                                                                               \
    MD_LAUNCH("cache4_score", st, (cache4_score_kernel<D_, F_>), dim3(B * H * tiles, chunks), 256, 0, A, FastDiv::make(tiles), FastDiv::make(H))
    if (d == 128) { if (dtype == MD_F32) MD_C4_SCORE(128, true); else MD_C4_SCORE(128, false); }
    else { if (dtype == MD_F32) MD_C4_SCORE(64, true); else MD_C4_SCORE(64, false); }
#undef MD_C4_SCORE
    MD_LAUNCH("cache4_choose", st, (cache4_choose_kernel), B * H * N, 256, 0, A, FastDiv::make(N), FastDiv::make(H));
    return check_launch(who);
}

struct ChosenPlan {
    C4Chosen cut;
    Parts parts;
    int tiles, waves;
    long units;
    size_t lds, bytes;
};
ChosenPlan chosen_plan(void* workspace, bool f32, int B, int N, int Hq, int d, int budget, const Pool& p) {
    ChosenPlan a;
    const int G = Hq / p.H, few = G < 16 ? G : 16;
    a.tiles = (G + 15) / 16;
    a.units = (long)B * N * p.H * a.tiles;
    a.cut = c4_chosen(a.units, budget, p.page);
    a.waves = 4;
    const size_t join = sizeof(float) * ((size_t)a.waves * few * (d + 4) + 2 * a.waves * 16), ring = (size_t)a.waves * kRing * (32 * d + 256);
    a.lds = (size_t)(a.cut.most + 1) / 2 * 16 + (join > ring ? join : ring);
    Carver c(workspace);
    const size_t places = a.cut.splits > 1 ? (size_t)a.units * a.cut.splits * 16 : 0;
    a.parts.o = c.take<float>(places * d);
    a.parts.ml = c.take<float2>(places);
    a.parts.blocks = a.parts.least = 0;
    a.bytes = c.off > 256 ? c.off : 256;
    (void)f32;
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
    const size_t x = chosen_plan(nullptr, false, B, N, Hq, d, budget, p).bytes, y = chosen_plan(nullptr, true, B, N, Hq, d, budget, p).bytes;
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
    const ChosenPlan plan = chosen_plan(workspace, dtype == MD_F32, B, N, Hq, d, budget, p);
    const size_t need = attend_chosen_bytes(B, N, Hq, H, d, budget, page);
    const Range r[] = {{out, rows_bytes(ol, B, N, Hq, d, dtype)}, {lse, lse ? (size_t)B * Hq * N * 4 : 0}, {workspace, workspace ? need : 0},
                       {q, rows_bytes(ql, B, N, Hq, d, dtype)}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {q_len, q_len ? (size_t)B * 4 : 0}, {keep, keep ? (size_t)B * max_pages * page : 0}, {chosen, (size_t)B * N * H * budget * 4}};
    rc = check_apart(who, r, 3, 10);
    if (rc != MD_OK) return rc;
    if (!workspace || workspace_bytes < need)
        return fail(MD_EWORKSPACE, "cache4_attend_chosen: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(MD_EALIGN, "cache4_attend_chosen: workspace must be 256-byte aligned");
    const AttendArgs A{q, static_cast<const uint8_t*>(cache), table, len, q_len, keep, out, lse, p, AttendDims{B, N, Hq / H, plan.tiles}, softmax_scale, ql, ol};
    const Chosen C{chosen, budget, plan.cut.splits, plan.cut.most};
    const int blocks = (int)(plan.units * plan.cut.splits);
    const bool stream_once = pool_bytes(p) > (size_t)128 << 20;
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_CHOSEN(D_, F_, S_)                                                                                                          \
    do {                                                                                                                                  \
        MD_LAUNCH("cache4_attend_chosen", st, (cache4_attend_chosen_kernel<D_, F_, S_>), blocks, plan.waves * 64, plan.lds, A, C, plan.parts); \
        if (C.splits > 1) MD_LAUNCH("cache4_chosen_join", st, (cache4_attend_chosen_join_kernel<D_, F_>), (int)plan.units, 256, 0, A, C, plan.parts); \
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
