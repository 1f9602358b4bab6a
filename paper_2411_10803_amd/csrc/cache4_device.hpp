// The cache held in 4 bits, on the device: numbers and their conversions, and the attention of a wave over pages, whichever they are.
#pragma once
#include "md_device.hpp"
#include "md_host.hpp"
#include "cache4_plan.hpp"

namespace md {
namespace {

constexpr float kLog2eC = 1.4426950408889634f, kLn2C = 0.6931471805599453f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Pool {
    int n_pages, page, page_shift, max_pages, H;
    long stride;                                     // bytes of one page and head
};

__device__ __forceinline__ uint32_t as_u32(bf16x2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float scale_of(uint32_t code) { return __uint_as_float(code << 23); }   // (255: read as NaN by the conversions)

// A lane's share of a row: d/16 channels, fp32.
template <int D, bool F32>
__device__ __forceinline__ void load_part(const void* base, long at, float (&x)[D / 16]) {
    constexpr int C = D / 16;
    if (F32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + at);
#pragma unroll
        for (int i = 0; i < C / 4; ++i) {
            const f32x4 w = p[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = w[j];
        }
    } else {
        uint32_t w[C / 2];
        if (D == 128) {
            const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at);
            const u32x4 v = *p;
#pragma unroll
            for (int i = 0; i < C / 2; ++i) w[i] = v[i];
        } else {
            const u32x2* p = reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(base) + at);
            const u32x2 v = *p;
#pragma unroll
            for (int i = 0; i < C / 2; ++i) w[i] = v[i];
        }
#pragma unroll
        for (int i = 0; i < C / 2; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    }
}

// Codes of a lane's d/16 channels (two to a byte) and the scale byte of the group that it shares with its neighbours.
template <int D>
__device__ __forceinline__ uint32_t quantise_part(const float (&x)[D / 16], int& code) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    most = max(most, (uint32_t)dpp_i<0xB1>((int)most, (int)most));
    most = max(most, (uint32_t)dpp_i<0x4E>((int)most, (int)most));
    if (D == 64) most = max(most, (uint32_t)dpp_i<0x141>((int)most, (int)most));
    code = c4_scale_code(most);
    const float s = scale_of(code);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    if (D == 128) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[D / 32], x[D / 32 + 1], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[D / 32 + 2], x[D / 32 + 3], s, 3);
    }
    return w;
}

template <int D>
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t w) {
    if (D == 128) *reinterpret_cast<uint32_t*>(p) = w;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w;
}

// ------------------------------------------------------------------------------------------------ attention

constexpr int kRing = 2;                         // steps that a wave of the attention has on their way
struct AttendDims { int B, N, G, tiles; };       // G: query heads of a K/V head; tiles: of query rows, in the longest case

struct AttendArgs {
    const void* q;
    const uint8_t* cache;
    const int32_t *table, *len, *q_len;
    const uint8_t* keep;
    void* out;
    float* lse;
    Pool p;
    AttendDims dim;
    float scale;
    KvLayout ql, ol;
};

// Sums over a part of a unit's keys: tile rows of d channels, and the (maximum, sum) pairs.
struct Parts {
    float* o;                                        // [2 * blocks][tile rows][d]
    float2* ml;                                      // [2 * blocks][tile rows]
    int blocks, least;
};

#define MD_VM_WAIT(n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory")
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const __attribute__((address_space(1))) void* global_ptr_t;

constexpr float kNoKey = -3.0e38f;                   // running maximum before the first key (below every score that matters)
// A running maximum may lag behind by this much (base 2) before the sums are scaled anew: probabilities up to 2^8 cost no accuracy.
constexpr float kLag = 8.f;
// A running maximum m is a rounded product of a score and the scale, and score * scale - m in one fma has that rounding in it: half a unit in
// the last place of m, which every probability of the row is off by as a power of two, in numerator and sum alike.  Up to here that
// is 2^4 at most; beyond 2^31 it would be more than fp32 holds, and the product is rounded as the maximum was.
constexpr float kFar = 67108864.f;

__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float s, int byte) {       // byte: a constant
    switch (byte) {
        case 0: return as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
        case 1: return as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        case 2: return as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
        default: return as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    }
}

// Two fp32 numbers as sums of bf16 parts, packed: two parts carry 16 bits, three carry all 24.
template <int TERMS>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&part)[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        part[i] = as_u32(__builtin_convertvector(f32x2{x, y}, bf16x2));
        if (i + 1 < TERMS) { x -= bf16_lo(part[i]); y -= bf16_hi(part[i]); }
    }
}

// A product that no addition is fused with.
__device__ __forceinline__ float rounded_product(float x, float y) {
    float r = x * y;
    asm("" : "+v"(r));
    return r;
}

// The larger of a value over the four lanes of one query (lane ^ 16, lane ^ 32), and the sum.
__device__ __forceinline__ float max_over_groups(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float sum_over_groups(float v) {
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}

// A pointer to global memory.  (One that comes out of argument() below is any pointer to the compiler, whose accesses then wait for LDS too.)
template <class T>
__device__ __forceinline__ __attribute__((address_space(1))) T* global(T* p) { return reinterpret_cast<__attribute__((address_space(1))) T*>(reinterpret_cast<uintptr_t>(p)); }
typedef const __attribute__((address_space(1))) uint8_t* bytes_t;
template <class T>
__device__ __forceinline__ T load_as(bytes_t p) { return *reinterpret_cast<const __attribute__((address_space(1))) T*>(p); }

// Numbers that a whole wave wants and that no kernel here writes while one reads them: by the constant address space, which makes
// the load a scalar one.  (As a vector load it would be waited for together with the keys on their way, which are younger.)
typedef const __attribute__((address_space(4))) int32_t* uniform_ptr_t;
__device__ __forceinline__ uniform_ptr_t uniform(const void* p) { return reinterpret_cast<uniform_ptr_t>(reinterpret_cast<uintptr_t>(p)); }

// The kernel's arguments, read again: what only the beginning and the end of a unit want does not take scalar registers
// while the keys go by (kept from the kernel's start on, 98 of them went through lanes of vector registers and back, step by step).
template <class T>
__device__ __forceinline__ T argument(int at) {
    uintptr_t p = (uintptr_t)__builtin_amdgcn_kernarg_segment_ptr() + at;
    asm volatile("" : "+s"(p));
    int32_t w[sizeof(T) / 4];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) w[i] = reinterpret_cast<uniform_ptr_t>(p)[i];
    T r;
    __builtin_memcpy(&r, w, sizeof(T));
    return r;
}
constexpr int kPartsAt = (sizeof(AttendArgs) + 7) / 8 * 8;

// What the entries of one sample look like to a call.
struct Sample { int b, length, nq; };
__device__ __forceinline__ Sample sample_of(const AttendArgs& A, int b) {
    Sample s;
    s.b = b;
    s.length = c4_clamp(uniform(A.len)[b], 0, A.p.max_pages << A.p.page_shift);
    s.nq = A.q_len ? c4_clamp(uniform(A.q_len)[b], 0, A.dim.N) : A.dim.N;
    return s;
}

// What a walk over the keys of one (sample, K/V head) needs.
struct Walk {
    bytes_t base;                                    // of the head in page 0
    uniform_ptr_t row, keep;                         // of the block table; of the mask, or null
    uint32_t pitch;                                  // 64-byte units from page to page
    int n_pages, page, page_shift, last_page;        // of the pool; tokens of a page; the table's last entry
    int end, level;                                  // keys that any row sees; that all rows see, but for those that a mask leaves out
    float c;                                         // softmax scale, base 2
};
struct Pages { int id[2]; };                         // of a step's two 16-key tiles
struct Kept { uint32_t w[2][4]; };                   // `keep` of a step's keys

// What the block table alone takes, so that its first entries can be asked for before the sample's length is there.
__device__ __forceinline__ Walk table_of(const AttendArgs& A, int b) {
    Walk w;
    w.row = uniform(A.table + (long)b * A.p.max_pages);
    w.page_shift = A.p.page_shift;
    w.last_page = A.p.max_pages - 1;
    return w;
}
// rows: the first and the last one that count, of those that the sample and head have
__device__ __forceinline__ void walk_of(Walk& w, const AttendArgs& A, const Sample& s, int h, int first_row, int last_row) {
    w.base = global(A.cache) + h * A.p.stride;
    w.keep = A.keep ? uniform(A.keep + (long)s.b * (A.p.max_pages << A.p.page_shift)) : nullptr;
    w.pitch = (uint32_t)(A.p.H * A.p.stride / 64);
    w.n_pages = A.p.n_pages;
    w.page = A.p.page;
    w.end = min(max(s.length - s.nq + last_row / A.dim.G + 1, 0), s.length);
    w.level = min(max(s.length - s.nq + first_row / A.dim.G + 1, 0), w.end);
    w.c = A.scale * kLog2eC;
}
// The entries as they stand in the table, which nobody looks at yet: a wave that asks for them a step ahead does not wait for them.
__device__ __forceinline__ Pages pages_at(const Walk& w, int step) {
    Pages r;
#pragma unroll
    for (int u = 0; u < 2; ++u) r.id[u] = w.row[min((step * 32 + 16 * u) >> w.page_shift, w.last_page)];
    return r;
}
// Those of a wave's first steps, on their way together with the sample's length: 0.3 us of a short unit's 10.
struct Early { Pages at[kRing + 1]; };
template <class W>
__device__ __forceinline__ Early early_pages(const W& w, int first, int stride) {
    Early r;
#pragma unroll
    for (int x = 0; x <= kRing; ++x) r.at[x] = pages_at(w, first + x * stride);
    return r;
}
__device__ __forceinline__ void arrived(Early& r, int& a, int& b) {
    static_assert(kRing == 2);
    asm volatile("" : "+s"(r.at[0].id[0]), "+s"(r.at[0].id[1]), "+s"(r.at[1].id[0]), "+s"(r.at[1].id[1]), "+s"(r.at[2].id[0]), "+s"(r.at[2].id[1]), "+s"(a), "+s"(b));
}
// Whether they name pages that the step needs.
__device__ __forceinline__ bool there(const Walk& w, int step, const Pages& p, int u) {
    return step * 32 + 16 * u < w.end && c4_page_id(p.id[u], w.n_pages) >= 0;
}
__device__ __forceinline__ bool hole(const Walk& w, int step, const Pages& p) { return !(there(w, step, p, 0) && there(w, step, p, 1)); }
// A step's pages where only whether they are there is of interest, and where their numbers are.
__device__ __forceinline__ Pages pages_for_mask(const Walk& w, int step) { return pages_at(w, step); }
__device__ __forceinline__ Pages pages_by_number(const Walk&, int, const Pages& p) { return p; }
// (page 0 is read in the place of one that is not there, and masked)
__device__ __forceinline__ bytes_t page_base(const Walk& w, int id) {
    return w.base + ((uint64_t)(((uint32_t)id < (uint32_t)w.n_pages ? (uint32_t)id : 0u) * w.pitch) << 6);
}
__device__ __forceinline__ Kept kept_at(const Walk& w, int step) {
    Kept r;
    if (w.keep) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = min(step * 8 + 4 * u, ((w.last_page + 1) << w.page_shift) / 4 - 4);       // (of a tile within the mask; any will do behind the end)
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
// Whether the mask leaves an entry out.
__device__ __forceinline__ bool left_out(const Walk& w, int t) { return w.keep && ((w.keep[t >> 2] >> (8 * (t & 3))) & 0xFF) == 0; }

// Whether some row does not see a page of a step that others see; all ones for those of a step's two tiles that the lane's row sees.
struct Sight { uint32_t u[2]; };
__device__ __forceinline__ bool uneven(const Walk&, int) { return false; }
__device__ __forceinline__ Sight sight_at(const Walk&, int) { return Sight{{0xFFFFFFFFu, 0xFFFFFFFFu}}; }

// 16 NT query rows of one (sample, K/V head) in a wave: queries, running maxima and sums.  Row r = i * G + g is the g-th query head
// of the K/V head at token i.
//
// S^T = K Q^T stands in the 16x16 accumulators (lane: query n = lane % 16, keys 4 b + 0..3 with b = lane / 16), so the
// probabilities are at once the right-hand operand of O^T = V^T P^T: with two 16-key tiles the eight contraction places of lane
// group b are keys 4 b + 0..3 of either tile.  The pages hold V so that a lane loads those keys' codes of its channels, and of K so
// that a lane loads d/4 channels of one token: from the loads to the matrix products no lane needs another's data.
// (The scaled 16x16x128 product would take K's codes and scales as they lie and a query as two e4m3 rows, a prompt's piece 7 % faster, but its sums
// are not fp32 ones: lse was off 10 to 40 times as far.)
template <int D, bool F32, int NT>
struct Rows {
    static constexpr int QT = F32 ? 3 : 1;           // bf16 parts of a query: fp32 has 24 bits
    static constexpr int PT = F32 ? 3 : 2;           // of a probability in the product with V: in one part its rounding would be as large as the
                                                     // output's (and 4 x 512 tokens of 32 heads on 8, up to 5888 keys, 193 us instead of 235)
    static constexpr int KS = D / 32;                // contraction steps of S
    static constexpr int J = D / 16;                 // 16-channel tiles of O

    bf16x8 q[NT][KS][QT];
    float m[NT], l[NT];
    f32x4 o[NT][J];
    int limit[NT];                                   // keys that the lane's row sees: up to its own position
    int n, lb;
    // What a probability's exponent is made of: score * by - off.  The scale to base 2 and the running maximum; once a maximum of the wave is
    // beyond kFar, 1 and 0, and the scores of every step are made the exponents themselves where the maxima are looked after (`lag` then lets no step by).
    float off[NT], by, lag;

    __device__ __forceinline__ void begin(const AttendArgs& A, const Sample& s, int h, int r0) {
        n = lane_id() & 15;
        lb = lane_id() >> 4;
        by = A.scale * kLog2eC;
        lag = kLag;
        const int G = A.dim.G, live = s.nq * G;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = r0 + 16 * t + n, i = r / G, hq = h * G + (r - i * G);
            limit[t] = r < live ? min(max(s.length - s.nq + i + 1, 0), s.length) : 0;
            m[t] = off[t] = kNoKey;
            l[t] = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KS; ++y) {
                uint32_t w[QT][4] = {};
                if (r < live) {
                    const long at = (long)s.b * A.ql.batch + (long)i * A.ql.token + (long)hq * A.ql.head + lb * (D / 4) + y * 8;
                    if (F32) {
                        const bytes_t from = reinterpret_cast<bytes_t>(global(static_cast<const float*>(A.q)) + at);
                        const f32x4 x[2] = {load_as<f32x4>(from), load_as<f32x4>(from + 16)};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t part[QT];
                            split_pair<QT>(x[j >> 1][2 * (j & 1)], x[j >> 1][2 * (j & 1) + 1], part);
#pragma unroll
                            for (int z = 0; z < QT; ++z) w[z][j] = part[z];
                        }
                    } else {
                        const u32x4 v = load_as<u32x4>(reinterpret_cast<bytes_t>(global(static_cast<const uint16_t*>(A.q)) + at));
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[0][j] = v[j];
                    }
                }
#pragma unroll
                for (int z = 0; z < QT; ++z) q[t][y][z] = __builtin_bit_cast(bf16x8, u32x4{w[z][0], w[z][1], w[z][2], w[z][3]});
            }
        }
    }

    // Whether a scale of V is beyond 252 in any lane: its numbers may not be finite.
    __device__ __forceinline__ static bool far(const uint32_t (&vs)[2]) {
        uint32_t r = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) r |= ((vs[u] & 0x7F7F7F7Fu) + 0x03030303u) & vs[u] & 0x80808080u;
        return __any(r != 0);
    }

    // Keys of the step that the call leaves out for all rows get a V scale of 1 (0 * NaN would count); `hides` gets a bit for each
    // of the lane's eight keys that its row does not see: of key x of tile u bit 8 x + 7 - 4 u.  Four keys at a time, a byte each.
    template <class W>
    __device__ __forceinline__ void mask(const W& w, int step, const Kept& kp, uint32_t (&vs)[2], uint32_t (&hides)[NT]) {
        constexpr uint32_t kTops = 0x80808080u;
        const auto nonzero = [](uint32_t x) { return (((x & ~kTops) + ~kTops) | x) & kTops; };
        const auto first = [](int n) { return n <= 0 ? 0u : kTops >> (32 - 8 * min(n, 4)); };
        const Pages known = pages_for_mask(w, step);
        const bool ok[2] = {there(w, step, known, 0), there(w, step, known, 1)};
        const Sight sight = sight_at(w, step);
        // (with a mask most steps are; without one a step comes here for its edge.  us, so / without `w.keep`: 4 x 512 tokens of 32 heads on 8, up to
        // 5888 keys 199.1 / 200.2, 4 x 2048 first ones 272.2 / 273.7; with a mask 238.5 / 240.1)
        const bool inside = w.keep && step * 32 + 32 <= w.level && ok[0] && ok[1];
        uint32_t on[2];
#pragma unroll
        for (int t = 0; t < NT; ++t) hides[t] = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = step * 32 + 16 * u + 4 * lb;
            const uint32_t w0 = kp.w[u][0], w1 = kp.w[u][1], w2 = kp.w[u][2], w3 = kp.w[u][3];
            const uint32_t even = lb & 2 ? w2 : w0, odd = lb & 2 ? w3 : w1, kept = lb & 1 ? odd : even;
            on[u] = nonzero(kept);
            if (inside) {
#pragma unroll
                for (int z = 0; z < NT; ++z) hides[z] |= (on[u] & (limit[z] > 0 ? sight.u[u] : 0u)) >> (4 * u);
            } else {
                on[u] &= first((ok[u] ? w.end : 0) - t);
#pragma unroll
                for (int z = 0; z < NT; ++z) hides[z] |= (on[u] & first(limit[z] - t) & sight.u[u]) >> (4 * u);
            }
        }
#pragma unroll
        for (int z = 0; z < NT; ++z) hides[z] = ~hides[z];
        if (!far(vs)) return;                        // (what is finite counts as 0 where its probability is)
        uint32_t nan = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t nans = kTops & ~nonzero(~vs[u]);
            nan |= on[u] & nans;
            const uint32_t out = (kTops & ~on[u]) | nans, bytes = (out << 1) - (out >> 7);
            vs[u] = (vs[u] & ~bytes) | (bytes & 0x7F7F7F7Fu);
        }
        // A NaN in V of a key that some rows see and others do not: the rows that see it get it in that group's channels here.
        if (__any(nan != 0)) {
            const Pages pg = pages_by_number(w, step, known);
#pragma unroll
            for (int z = 0; z < NT; ++z) {
                float poison = 0.f;
#pragma unroll 1
                for (int x = 0; x < 32; ++x) {
                    const int t = step * 32 + x, id = x < 16 ? pg.id[0] : pg.id[1];
                    if (!(x < 16 ? ok[0] : ok[1]) || t >= w.end || left_out(w, t)) continue;
                    if (t < limit[z] && (x < 16 ? sight.u[0] : sight.u[1]) && page_base(w, id)[c4_v_scales(w.page, t & (w.page - 1), lb * D / 128, D)] == 255) poison = __builtin_nanf("");
                }
#pragma unroll
                for (int j = 0; j < J; ++j) o[z][j] += poison;
            }
        }
    }

    // Scores of pages that the lane's row does not see.
    __device__ __forceinline__ static void hide_pages(f32x4 (&st)[NT][2], const Sight& sight) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (!sight.u[x >> 2]) st[t][x >> 2][x & 3] = -INFINITY;
    }
    // Scores of keys that the lane's row does not see.
    __device__ __forceinline__ static void hide(f32x4 (&st)[NT][2], uint32_t (&hides)[NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            asm volatile("" : "+v"(hides[t]));       // (its bits are looked at here, and not in the steps that need no mask)
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if ((hides[t] >> (8 * (x & 3) + 7 - 4 * (x >> 2))) & 1) st[t][x >> 2][x & 3] = -INFINITY;
        }
    }

    // Probabilities of tile t's scores, in PT parts; the running maximum follows where the scores have outgrown it.
    __device__ __forceinline__ void softmax(int t, f32x4 (&st)[2], float c, bf16x8 (&p)[PT]) {
        float most = st[0][0];
#pragma unroll
        for (int x = 1; x < 8; ++x) most = fmaxf(most, st[x >> 2][x & 3]);
        most *= c;
        if (__any(most > m[t] + lag)) {
            const float m2 = fmaxf(m[t], max_over_groups(most)), a = fast_exp2(m[t] - m2);
            m[t] = off[t] = m2;
            l[t] *= a;
#pragma unroll
            for (int j = 0; j < J; ++j) o[t][j] *= a;
            if (lag < 0.f || __any(fabsf(m2) > kFar && m2 > kNoKey)) {
                lag = -INFINITY;
                by = 1.f;
#pragma unroll
                for (int z = 0; z < NT; ++z) off[z] = 0.f;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const float s = st[x >> 2][x & 3], near = fmaf(s, c, -m2), beyond = rounded_product(s, c) - m2;
                    st[x >> 2][x & 3] = fabsf(m2) > kFar ? beyond : near;
                }
            }
        }
        uint32_t w[PT][4];
#pragma unroll
        for (int x = 0; x < 8; x += 2) {
            const float p0 = fast_exp2(fmaf(st[x >> 2][x & 3], by, -off[t])), p1 = fast_exp2(fmaf(st[x >> 2][(x & 3) + 1], by, -off[t]));
            l[t] += p0 + p1;
            uint32_t part[PT];
            split_pair<PT>(p0, p1, part);
#pragma unroll
            for (int z = 0; z < PT; ++z) w[z][x / 2] = part[z];
        }
#pragma unroll
        for (int z = 0; z < PT; ++z) p[z] = __builtin_bit_cast(bf16x8, u32x4{w[z][0], w[z][1], w[z][2], w[z][3]});
    }
};

// A wave that brings its own keys: steps of 32, straight from the pages.
template <int D, bool F32, int NT, bool STREAM>
struct Sweep : Rows<D, F32, NT> {
    typedef Rows<D, F32, NT> R;
    using R::KS; using R::J; using R::QT; using R::PT; using R::n; using R::lb; using R::q; using R::o;
    static constexpr int RING = kRing;               // steps on their way
    static constexpr int LOADS = D == 128 ? 5 : 3;   // load instructions of a step
    static constexpr int CODES = 32 * D, SLOT = CODES + 256;     // bytes of a step's codes; of its place in LDS
    static constexpr int KB = D / 8;                 // bytes of codes that a lane works on of a token's K, and of four tokens' V

    struct Keys { uint32_t k[2][KB / 4], v[2][KB / 4], ks[2], vs[2]; };      // of one step

    uint32_t at_k, at_v, at_s;                       // the byte offsets that the lane loads from, from its tile's place in a page on
    bool second;                                     // the lane loads scales of the second tile

    __device__ __forceinline__ void begin(const AttendArgs& A, const Sample& s, int h, int r0) {
        R::begin(A, s, h, r0);
        const int lane = lane_id(), half = D == 128 ? lane : lane & 31;
        at_k = D == 128 ? c4_k_codes(n, D) + lb * KB : half * 16;
        at_v = D == 128 ? c4_v_codes(A.p.page, 4 * lb, n, D) : c4_v_codes(A.p.page, 0, 0, D) + half * 16;
        constexpr int W = D / 8;                     // words of a tile's scales of K; as many of V (d = 64: lanes from 32 on repeat)
        const int word = lane & (4 * W - 1);
        second = (word / W) & 1;
        at_s = (word < 2 * W ? c4_k_scales(A.p.page, 0, D) : c4_v_scales(A.p.page, 0, 0, D)) + (word % W) * 4;
    }

    // Asks for a step's keys: loads that write LDS directly, SLOT bytes at `slot` (the wave's own).  They are a queue and nothing else: what
    // a lane works with lies where the loads put it, and a wave has RING steps on their way without a register for them.
    //   d = 128: a lane's 16 bytes of K and of V, tile by tile;  d = 64: the tiles' 512 bytes of K as they are, and of V
    //   then the scales: 16 keys' bytes of K of the first and the second tile, then V's
    __device__ __forceinline__ void ask(const Walk& w, int step, const Pages& pg, char* slot) const {
        const int at = (step * 32) & (w.page - 1);
        bytes_t base[2];
        int place[2] = {at, at + 16};
        base[0] = base[1] = page_base(w, pg.id[0]);
        if (w.page_shift == 4) {                     // (other pages hold both tiles)
            place[1] = 0;
            base[1] = page_base(w, pg.id[1]);
        }
        if (D == 128) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                to_lds<16>(base[u] + place[u] * (D / 2) + at_k, slot + u * 1024);
                to_lds<16>(base[u] + place[u] * (D / 2) + at_v, slot + 2048 + u * 1024);
            }
        } else {
            const bytes_t codes = lane_id() < 32 ? base[0] + place[0] * (D / 2) : base[1] + place[1] * (D / 2);
            to_lds<16>(codes + at_k, slot);
            to_lds<16>(codes + at_v, slot + 1024);
        }
        to_lds<4>((second ? base[1] + place[1] * (D / 32) : base[0] + place[0] * (D / 32)) + at_s, slot + CODES);
    }
    template <int BYTES>
    __device__ static __forceinline__ void to_lds(bytes_t from, char* to) {
        const global_ptr_t g = reinterpret_cast<global_ptr_t>(from);
        if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds(g, (lds_ptr_t)to, 16, 0, STREAM ? 2 : 0);
        else __builtin_amdgcn_global_load_lds(g, (lds_ptr_t)to, 4, 0, STREAM ? 2 : 0);
    }
    // The keys of a step out of its slot: returns once they are in registers, and the slot is free.
    __device__ __forceinline__ Keys take(const char* slot) const {
        Keys r;
        const uint32_t at = (uint32_t)(uintptr_t)(lds_ptr_t)const_cast<char*>(slot);
        if constexpr (D == 128) {
            u32x4 k0, k1, v0, v1;
            asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:1024\n\tds_read_b128 %2, %8 offset:2*1024\n\tds_read_b128 %3, %8 offset:3*1024\n\t"
                         "ds_read_u8 %4, %9 offset:4096\n\tds_read_u8 %5, %9 offset:4160\n\tds_read_b32 %6, %10 offset:4224\n\tds_read_b32 %7, %10 offset:4288\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(k0), "=&v"(k1), "=&v"(v0), "=&v"(v1), "=&v"(r.ks[0]), "=&v"(r.ks[1]), "=&v"(r.vs[0]), "=&v"(r.vs[1])
                         : "v"(at + lane_id() * 16), "v"(at + n * 4 + lb), "v"(at + (lb * 4 + (n >> 2)) * 4) : "memory");
#pragma unroll
            for (int x = 0; x < 4; ++x) { r.k[0][x] = k0[x]; r.k[1][x] = k1[x]; r.v[0][x] = v0[x]; r.v[1][x] = v1[x]; }
        } else {
            u32x2 k0, k1, v0, v1;
            asm volatile("ds_read_b64 %0, %8\n\tds_read_b64 %1, %8 offset:512\n\tds_read_b64 %2, %9\n\tds_read_b64 %3, %9 offset:512\n\t"
                         "ds_read_u8 %4, %10 offset:2048\n\tds_read_u8 %5, %10 offset:2080\n\tds_read_b32 %6, %11 offset:2112\n\tds_read_b32 %7, %11 offset:2144\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(k0), "=&v"(k1), "=&v"(v0), "=&v"(v1), "=&v"(r.ks[0]), "=&v"(r.ks[1]), "=&v"(r.vs[0]), "=&v"(r.vs[1])
                         : "v"(at + n * 32 + lb * 8), "v"(at + 1024 + lane_id() * 8), "v"(at + n * 2 + (lb >> 1)), "v"(at + (lb * 2 + (n >> 3)) * 4)
                         : "memory");
#pragma unroll
            for (int x = 0; x < 2; ++x) { r.k[0][x] = k0[x]; r.k[1][x] = k1[x]; r.v[0][x] = v0[x]; r.v[1][x] = v1[x]; }
        }
        return r;
    }

    __device__ __forceinline__ void step(const Walk& w, const Keys& K, bool masked, uint32_t (&hides)[NT], bool pages, const Sight& sight) {
        f32x4 st[NT][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float ks = scale_of(K.ks[u]);
#pragma unroll
            for (int t = 0; t < NT; ++t) st[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KS; ++y) {
                const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{fp4_pair(K.k[u][y], ks, 0), fp4_pair(K.k[u][y], ks, 1),
                                                                  fp4_pair(K.k[u][y], ks, 2), fp4_pair(K.k[u][y], ks, 3)});
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int z = QT - 1; z >= 0; --z) st[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[t][y][z], st[t][u], 0, 0, 0);
            }
        }
        if (masked) R::hide(st, hides);
        if (pages) R::hide_pages(st, sight);
        bf16x8 p[NT][PT];
#pragma unroll
        for (int t = 0; t < NT; ++t) R::softmax(t, st[t], w.c, p[t]);
        // V^T P^T: byte y of a token's share is channels 2 y and 2 y + 1 of this lane
#pragma unroll
        for (int y = 0; y < J / 2; ++y) {
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t f[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int at = x * (D / 32) + y; // byte of the lane's load
                    f[x] = fp4_pair(K.v[u][at / 4], scale_of((K.vs[u] >> (8 * x)) & 0xFF), at % 4);
                }
                lo[2 * u] = __builtin_amdgcn_perm(f[1], f[0], 0x05040100u);
                lo[2 * u + 1] = __builtin_amdgcn_perm(f[3], f[2], 0x05040100u);
                hi[2 * u] = __builtin_amdgcn_perm(f[1], f[0], 0x07060302u);
                hi[2 * u + 1] = __builtin_amdgcn_perm(f[3], f[2], 0x07060302u);
            }
            const bf16x8 vl = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], lo[2], lo[3]});
            const bf16x8 vh = __builtin_bit_cast(bf16x8, u32x4{hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int z = PT - 1; z >= 0; --z) {
                    o[t][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vl, p[t][z], o[t][2 * y], 0, 0, 0);
                    o[t][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, p[t][z], o[t][2 * y + 1], 0, 0, 0);
                }
        }
    }

    // Steps first, first + stride, .. below `stop` (of 32 keys).  `ring`: the wave's RING slots.
    template <class W>
    __device__ __forceinline__ void run(const W& w, int first, int stop, int stride, char* ring, const Early& early) {
        stop = min(stop, (w.end + 31) >> 5);
        if (first >= stop) return;
        uint32_t holes = 0;                                      // bit x: a page of the step in slot x is not there
#pragma unroll
        for (int x = 0; x < RING; ++x)
            if (first + x * stride < stop) {
                const Pages pg = early.at[x];
                if (hole(w, first + x * stride, pg)) holes |= 1u << x;
                ask(w, first + x * stride, pg, ring + x * SLOT);
            }
        // The queries are there from here on: a wait for them within the loop would be one for the keys on their way too, step by step.
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int y = 0; y < KS; ++y)
#pragma unroll
                for (int z = 0; z < QT; ++z) asm volatile("" : "+v"(q[t][y][z]));
        int x = 0;
        Pages next = early.at[RING];                             // (asked for a step before they are needed)
        Kept later = kept_at(w, first);
        for (int i = first; i < stop; i += stride) {
            const int ahead = i + RING * stride;
            const Pages pg = next;
            const Kept kp = later;
            if (ahead - stride < stop) { MD_VM_WAIT((RING - 1) * LOADS); } else { MD_VM_WAIT(0); }
            Keys k = take(ring + x * SLOT);
            __builtin_amdgcn_sched_barrier(0);                   // (what is asked for before the wait for LDS is waited for with it)
            next = pages_at(w, ahead + stride);
            later = kept_at(w, i + stride);
            bool masked = ((holes >> x) & 1) != 0 || w.keep || i * 32 + 32 > w.level, pages = false;
            holes &= ~(1u << x);
            if (ahead < stop) {
                if (hole(w, ahead, pg)) holes |= 1u << x;
                ask(w, ahead, pg, ring + x * SLOT);
            }
            x = x + 1 == RING ? 0 : x + 1;
            // (where nothing but whole pages is hidden, from some rows: without a mask, as long as V is finite)
            Sight sight{{0, 0}};
            if (!masked && uneven(w, i)) {
                pages = !R::far(k.vs);
                masked = !pages;
                if (pages) sight = sight_at(w, i);
            }
            uint32_t hides[NT];
            if (masked) R::mask(w, i, kp, k.vs, hides);
            step(w, k, masked, hides, pages, sight);
        }
    }
};

// Writes one lane's share of a finished row: d/16 channels from `part` on.
template <int D, bool F32>
__device__ __forceinline__ void store_out(const AttendArgs& A, int b, int h, int r, int part, const float (&x)[D / 16], float m, float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;      // a row that sees no key: zeros
    const int G = A.dim.G, i = r / G, hq = h * G + (r - i * G);
    const long to = (long)b * A.ol.batch + (long)i * A.ol.token + (long)hq * A.ol.head + part * (D / 16);
    if (F32) {
        auto p = reinterpret_cast<__attribute__((address_space(1))) f32x4*>(global(static_cast<float*>(A.out)) + to);
#pragma unroll
        for (int j = 0; j < D / 64; ++j) p[j] = f32x4{x[4 * j] * inv, x[4 * j + 1] * inv, x[4 * j + 2] * inv, x[4 * j + 3] * inv};
    } else {
        auto p = reinterpret_cast<__attribute__((address_space(1))) uint32_t*>(global(static_cast<uint16_t*>(A.out)) + to);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) p[j] = as_u32(__builtin_convertvector(f32x2{x[2 * j] * inv, x[2 * j + 1] * inv}, bf16x2));
    }
    if (A.lse && part == 0) global(A.lse)[((long)b * A.p.H * G + hq) * A.dim.N + i] = l == 0.f ? -INFINITY : (m + fast_log2(l)) * kLn2C;
}
template <int D>
__device__ __forceinline__ void store_part(const Parts& parts, int place, int tile_rows, int row, int part, const float (&x)[D / 16], float m, float l) {
    auto p = reinterpret_cast<__attribute__((address_space(1))) f32x4*>(global(parts.o) + ((long)place * tile_rows + row) * D + part * (D / 16));
#pragma unroll
    for (int j = 0; j < D / 64; ++j) p[j] = f32x4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
    if (part == 0) *reinterpret_cast<__attribute__((address_space(1))) f32x2*>(global(parts.ml) + (long)place * tile_rows + row) = f32x2{m, l};
}

// A block's waves join their sums of 16 rows at a time through LDS: [waves][rows][D + 4] and the (m, l) pairs behind.  Then
// thread (row, part) calls done(row, part, x, m, l).
template <int D, int NT, class S, class Done>
__device__ __forceinline__ void join_waves(S& w, int rows, float* lds, Done done) {
    const int wv = wave_id(), nw = blockDim.x >> 6, tid = threadIdx.x, few = min(rows, 16);
    float* so = lds;
    float* sm = lds + nw * few * (D + 4);
    float* sl = sm + nw * 16;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (16 * t >= rows) return;
        if (t) __syncthreads();
        const float l = sum_over_groups(w.l[t]);
        if (w.n < few) {
            if (w.lb == 0) { sm[wv * 16 + w.n] = w.m[t]; sl[wv * 16 + w.n] = l; }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<f32x4*>(so + (wv * few + w.n) * (D + 4) + w.lb * (D / 4) + x * (D / 16) + j) =
                        f32x4{w.o[t][j][x], w.o[t][j + 1][x], w.o[t][j + 2][x], w.o[t][j + 3][x]};
        }
        __syncthreads();
        const int row = tid >> 4, part = tid & 15;
        if (row >= few || 16 * t + row >= rows) continue;
        float top = kNoKey, sum = 0.f, acc[D / 16] = {};
        for (int x = 0; x < nw; ++x) top = fmaxf(top, sm[x * 16 + row]);
        for (int x = 0; x < nw; ++x) {
            const float a = fast_exp2(sm[x * 16 + row] - top);
            sum = fmaf(sl[x * 16 + row], a, sum);
            const f32x4* from = reinterpret_cast<const f32x4*>(so + (x * few + row) * (D + 4) + part * (D / 16));
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                const f32x4 v = from[j];
#pragma unroll
                for (int y = 0; y < 4; ++y) acc[4 * j + y] = fmaf(v[y], a, acc[4 * j + y]);
            }
        }
        done(16 * t + row, part, acc, top, sum);
    }
}

}  // namespace
}  // namespace md
