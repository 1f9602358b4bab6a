// The cache held in 4 bits: block tables and slots from request lengths, rows in, rows out, and the attention that reads it.
//
// A group of 32 channels of one token and head is held as 32 four-bit floats (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6) with one power of two as scale: the form that gfx950 converts in hardware (v_cvt_scalef32_pk_*_fp4, two numbers
// per instruction, the scale applied on the way).  A scaled value is exact in bf16, so K and V reach the matrix cores without
// another rounding.
//
//   cache4_pages_kernel, cache4_slots_kernel   lengths -> pages taken and released, table entries, slots
//   cache4_write_kernel                        rows -> codes and scales, at their slots
//   cache4_read_kernel                         pages -> rows
//   cache4_attend_kernel                       softmax(scale Q K^T) V over the pages
#include "md_device.hpp"
#include "md_host.hpp"
#include "cache4_plan.hpp"

#include <cmath>

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

// ------------------------------------------------------------------------------------------------ pages and slots

// One request's part of a call, handed from the first kernel to the second: lengths before and after, and the place on the
// stack of the first page that it takes.
struct PagePlan { int old_len, new_len, first; };

// One block: counts the pages that leave and come, puts the released ones on the stack, and gives each request its place on it.
// A chain of two scans over the requests; its time is that chain's (see cache4_pages_impl).
__global__ __launch_bounds__(1024) void cache4_pages_kernel(
    const int32_t* __restrict__ new_len, int32_t* __restrict__ len, const int32_t* __restrict__ table,
    int32_t* __restrict__ free_pages, int32_t* __restrict__ n_free, int32_t* __restrict__ missing,
    int B, int max_pages, int n_pages, int page_shift, PagePlan* __restrict__ plan)
{
    __shared__ int s_red[16];
    const int tid = threadIdx.x, top = c4_clamp(n_free[0], 0, n_pages);
    long leave = 0, come = 0;
    for (int b = tid; b < B; b += 1024) {
        const C4Change c = c4_change(len[b], new_len[b], max_pages, page_shift);
        if (c.held > c.need) leave += c.held - c.need;
        else come += c.need - c.held;
    }
    // (the host checks that B * max_pages fits 31 bits)
    const int R = block_sum_i((int)leave, s_red), T = block_sum_i((int)come, s_red);
    const int left = top + R - T;
    if (tid == 0) missing[0] = left < 0 ? -left : 0;
    if (left < 0) {
        for (int b = tid; b < B; b += 1024) plan[b] = PagePlan{0, 0, 0};
        return;
    }
    int left_before = 0, come_before = 0;
    for (int b0 = 0; b0 < B; b0 += 1024) {
        const int b = b0 + tid;
        C4Change c{0, 0, 0, 0};
        if (b < B) c = c4_change(len[b], new_len[b], max_pages, page_shift);
        const int lv = max(c.held - c.need, 0), cm = max(c.need - c.held, 0);
        int lt, ct;
        const int lp = left_before + block_exscan_i(lv, s_red, lt), cp = come_before + block_exscan_i(cm, s_red, ct);
        left_before += lt;
        come_before += ct;
        if (b >= B) continue;
        for (int e = 0; e < lv; ++e) {
            const int at = c4_released_at(top, R, lp + e);
            if (at < n_pages) free_pages[at] = table[(long)b * max_pages + c.need + e];
        }
        plan[b] = PagePlan{c.old_len, c.new_len, c4_taken_at(top, R, cp)};
        len[b] = c.new_len;
    }
    if (tid == 0) n_free[0] = min(left, n_pages);
}

// Entries and slots of one request per blockIdx.y.
__global__ __launch_bounds__(256) void cache4_slots_kernel(
    const PagePlan* __restrict__ plan, int32_t* __restrict__ table, const int32_t* __restrict__ free_pages,
    int32_t* __restrict__ slots, int max_pages, int n_pages, int page_shift, int N)
{
    const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    const PagePlan p = plan[b];
    const int held = c4_pages_of(p.old_len, page_shift), need = c4_pages_of(p.new_len, page_shift);
    int32_t* row = table + (long)b * max_pages;
    // place `first - j` of the stack holds the j-th page that the request takes
    if (i < need - held && p.first - i >= 0 && p.first - i < n_pages) row[held + i] = free_pages[p.first - i];
    if (slots && i < N) {
        const int at = p.old_len + i;
        int slot = -1;
        if (at < p.new_len) {
            const int e = at >> page_shift, j = p.first - (e - held);
            const int id = c4_page_id(e < held ? row[e] : (j >= 0 && j < n_pages ? free_pages[j] : -1), n_pages);
            if (id >= 0) slot = (int)(((uint32_t)id << page_shift) + (at & ((1 << page_shift) - 1)));
        }
        slots[(long)b * N + i] = slot;
    }
}

// ------------------------------------------------------------------------------------------------ rows in and out

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
        const u32x2* p = reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
        for (int i = 0; i < C / 4; ++i) {
            const u32x2 w = p[i];
            x[4 * i] = bf16_lo(w[0]); x[4 * i + 1] = bf16_hi(w[0]);
            x[4 * i + 2] = bf16_lo(w[1]); x[4 * i + 3] = bf16_hi(w[1]);
        }
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

// A wave writes four rows of one head: sixteen lanes per row, d/16 channels each.
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_write_kernel(
    const void* __restrict__ k_new, const void* __restrict__ v_new, const int32_t* __restrict__ slots, uint8_t* __restrict__ cache,
    Pool p, KvLayout lay, long rows, int N)
{
    const int lane = lane_id(), part = lane & 15;
    const long unit = (long)blockIdx.x * 4 + wave_id();
    const int h = (int)(unit % p.H);
    const long r = unit / p.H * 4 + (lane >> 4);
    C4Slot at{-1, 0};
    if (r < rows) at = c4_slot(slots[r], p.n_pages, p.page_shift);
    float k[D / 16] = {}, v[D / 16] = {};
    if (at.page >= 0) {
        const long b = r / N, from = b * lay.batch + (r - b * N) * lay.token + (long)h * lay.head + part * (D / 16);
        load_part<D, F32>(k_new, from, k);
        load_part<D, F32>(v_new, from, v);
    }
    int ks, vs;
    const uint32_t kw = quantise_part<D>(k, ks), vw = quantise_part<D>(v, vs);
    if (at.page < 0) return;
    uint8_t* to = cache + ((long)at.page * p.H + h) * p.stride;
    store_codes<D>(to + c4_k_codes(at.place, D) + part * (D / 32), kw);
    store_codes<D>(to + c4_v_codes(p.page, at.place, part, D), vw);
    const int group = part / (512 / D);
    if (part % (512 / D) == 0) {
        to[c4_k_scales(p.page, at.place, D) + group] = (uint8_t)ks;
        to[c4_v_scales(p.page, at.place, group, D)] = (uint8_t)vs;
    }
}

template <int D>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p) {
    return D == 128 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
}

template <int D, bool F32>
__device__ __forceinline__ void store_values(void* base, long at, uint32_t w, uint32_t code) {
    const float s = scale_of(code);
    if (F32) {
        f32x2* p = reinterpret_cast<f32x2*>(static_cast<float*>(base) + at);
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
        if (D == 128) {
            p[D / 64] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2);
            p[D / 64 + 1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
        }
    } else {
        uint32_t* p = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(base) + at);
        p[0] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
        p[1] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        if (D == 128) {
            p[D / 64] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
            p[D / 64 + 1] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
        }
    }
}

// The way back, shared out as in the write.
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_read_kernel(
    const uint8_t* __restrict__ cache, const int32_t* __restrict__ table, const int32_t* __restrict__ len, const int32_t* __restrict__ first,
    void* __restrict__ k_out, void* __restrict__ v_out, Pool p, KvLayout lay, long rows, int N)
{
    const int lane = lane_id(), part = lane & 15;
    const long unit = (long)blockIdx.x * 4 + wave_id();
    const int h = (int)(unit % p.H);
    const long r = unit / p.H * 4 + (lane >> 4);
    if (r >= rows) return;
    const int b = (int)(r / N), i = (int)(r - (long)b * N);
    const long at = (first ? (long)first[b] : 0l) + i;
    if (at < 0 || at >= c4_clamp(len[b], 0, p.max_pages << p.page_shift)) return;
    const int t = (int)at & (p.page - 1), id = c4_page_id(table[(long)b * p.max_pages + ((int)at >> p.page_shift)], p.n_pages);
    if (id < 0) return;
    const uint8_t* from = cache + ((long)id * p.H + h) * p.stride;
    const uint32_t kw = load_codes<D>(from + c4_k_codes(t, D) + part * (D / 32)), vw = load_codes<D>(from + c4_v_codes(p.page, t, part, D));
    const int group = part / (512 / D);
    const uint32_t ks = from[c4_k_scales(p.page, t, D) + group], vs = from[c4_v_scales(p.page, t, group, D)];
    const long to = b * lay.batch + i * lay.token + (long)h * lay.head + part * (D / 16);
    store_values<D, F32>(k_out, to, kw, ks);
    store_values<D, F32>(v_out, to, vw, vs);
}

// ------------------------------------------------------------------------------------------------ attention

struct AttendDims { int B, N, G, tiles; };           // G: query heads of a K/V head; tiles: of 16 query rows

constexpr float kNoKey = -3.0e38f;                   // running maximum before the first key (below every finite score that matters)

// fp32 as a sum of bf16 parts: two carry 16 bits, three carry all 24.
template <int TERMS>
__device__ __forceinline__ void split_bf16(float x, uint32_t (&part)[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        part[i] = f32_to_bf16(x);
        x -= __uint_as_float(part[i] << 16);
    }
}

// Sixteen query rows of one (sample, K/V head) per block, row r = i * G + g (token i, g-th query head of the K/V head); the
// waves of the block take the 32-key steps in turn and join their sums at the end.
//
// A wave holds S^T = K Q^T in the 16x16 accumulators (lane: query n = lane % 16, keys 4 b + 0..3 with b = lane / 16), so the
// probabilities are at once the right-hand operand of O^T = V^T P^T: with two 16-key tiles the eight contraction places of lane
// group b are keys 4 b + 0..3 of either tile.  The pages hold V so that a lane loads those keys' codes of its channels, and of K so
// that a lane loads d/4 channels of one token; nothing goes through LDS until the end.
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_attend_kernel(
    const void* __restrict__ q, const uint8_t* __restrict__ cache, const int32_t* __restrict__ table, const int32_t* __restrict__ len,
    const int32_t* __restrict__ q_len, const uint8_t* __restrict__ keep, Pool p, AttendDims dim, float scale,
    void* __restrict__ out, float* __restrict__ lse, KvLayout q_lay, KvLayout o_lay)
{
    constexpr int QT = F32 ? 3 : 1;                  // bf16 parts of a query: fp32 has 24 bits
    constexpr int PT = F32 ? 3 : 2;                  // of a probability: in one part its rounding would be as large as the output's
    constexpr int KS = D / 32;                       // contraction steps of S
    constexpr int J = D / 16;                        // 16-channel tiles of O
    constexpr int KB = D / 8;                        // bytes of codes a lane loads of a token's K, and of four tokens' V
    __shared__ float s_o[4][16][D + 4];
    __shared__ float s_m[4][16], s_l[4][16];
    const int lane = lane_id(), wv = wave_id(), n = lane & 15, lb = lane >> 4;
    const int tile = blockIdx.x % dim.tiles, bh = blockIdx.x / dim.tiles, h = bh % p.H, b = bh / p.H;
    const int cap = p.max_pages << p.page_shift;
    const int length = c4_clamp(len[b], 0, cap), nq = q_len ? c4_clamp(q_len[b], 0, dim.N) : dim.N;
    const int live = nq * dim.G;                     // query rows of this sample and head
    const int r0 = tile * 16;
    if (r0 >= live) return;
    const int r = r0 + n, i = r / dim.G, hq = h * dim.G + (r - i * dim.G);
    // keys that a row sees: up to its own position
    const int limit = r < live ? min(max(length - nq + i + 1, 0), length) : 0;
    const int last = min(r0 + 15, live - 1);
    const int end = min(max(length - nq + last / dim.G + 1, 0), length), full = max(length - nq + r0 / dim.G + 1, 0);

    bf16x8 qf[KS][QT];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        float x[8] = {};
        if (r < live) {
            const long at = (long)b * q_lay.batch + (long)i * q_lay.token + (long)hq * q_lay.head + lb * (D / 4) + s * 8;
            float y[8];
            load_part<128, F32>(q, at, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = y[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t part[QT];
            split_bf16<QT>(x[j], part);
#pragma unroll
            for (int t = 0; t < QT; ++t) qf[s][t][j] = __builtin_bit_cast(__bf16, (uint16_t)part[t]);
        }
    }

    const float c = scale * kLog2eC;
    float m = kNoKey, l = 0.f;
    f32x4 o[J];
#pragma unroll
    for (int j = 0; j < J; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int32_t* row = table + (long)b * p.max_pages;

    for (int t0 = wv * 32; t0 < end; t0 += 128) {
        const uint8_t* base[2];
        bool there[2];
        int place[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = t0 + 16 * u;
            const int id = t < end ? c4_page_id(__builtin_amdgcn_readfirstlane(row[t >> p.page_shift]), p.n_pages) : -1;
            there[u] = id >= 0;                      // (page 0 is read in the place of one that is not there, and masked)
            place[u] = t & (p.page - 1);
            base[u] = cache + ((long)max(id, 0) * p.H + h) * p.stride;
        }
        uint32_t kw[2][KB / 4], vw[2][KB / 4], ksc[2], vsc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint8_t* kp = base[u] + c4_k_codes(place[u] + n, D) + lb * KB;
            const uint8_t* vp = base[u] + c4_v_codes(p.page, place[u] + 4 * lb, n, D);
            if (D == 128) {
                const u32x4 a = *reinterpret_cast<const u32x4*>(kp), w = *reinterpret_cast<const u32x4*>(vp);
#pragma unroll
                for (int x = 0; x < KB / 4; ++x) { kw[u][x] = a[x]; vw[u][x] = w[x]; }
            } else {
                const u32x2 a = *reinterpret_cast<const u32x2*>(kp), w = *reinterpret_cast<const u32x2*>(vp);
#pragma unroll
                for (int x = 0; x < KB / 4; ++x) { kw[u][x] = a[x]; vw[u][x] = w[x]; }
            }
            ksc[u] = base[u][c4_k_scales(p.page, place[u] + n, D) + lb * D / 128];
            vsc[u] = *reinterpret_cast<const uint32_t*>(base[u] + c4_v_scales(p.page, place[u] + 4 * lb, n * D / 512, D));
        }
        // which of this lane's keys its query row sees
        uint32_t sees = 0xFF;
        const bool masked = !there[0] || !there[1] || t0 + 32 > full || t0 + 32 > end || keep;
        if (masked) {
            sees = 0;
            uint32_t drop = 0;                       // keys that no row sees: their V must not count, whatever it holds
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t kept = 0x01010101u;
                const int t = t0 + 16 * u + 4 * lb;
                if (keep && t < cap) kept = *reinterpret_cast<const uint32_t*>(keep + (long)b * cap + t);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const bool on = there[u] && t + x < end && ((kept >> (8 * x)) & 0xFF) != 0;
                    if (on && t + x < limit) sees |= 1u << (4 * u + x);
                    if (!on) drop |= 1u << (4 * u + x);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (drop & (1u << (4 * u + x))) vsc[u] &= ~(0xFFu << (8 * x));
            // A NaN in V of a key that some rows see and others do not: 0 * NaN would reach those too.  Its scale goes, and the
            // rows that do see it get the NaN in that group's channels by themselves.
            bool nan = false;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (((vsc[u] >> (8 * x)) & 0xFF) == 255) { nan = true; vsc[u] &= ~(0xFFu << (8 * x)); }
            if (__any(nan)) {
                float poison = 0.f;
                for (int x = 0; x < 32; ++x) {
                    const int u = x >> 4, t = t0 + x;
                    if (!there[u] || t >= limit || (keep && keep[(long)b * cap + t] == 0)) continue;
                    if (base[u][c4_v_scales(p.page, place[u] + (x & 15), lb * D / 128, D)] == 255) poison = __builtin_nanf("");
                }
#pragma unroll
                for (int j = 0; j < J; ++j) o[j] += poison;
            }
        }
        f32x4 st[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float s = scale_of(ksc[u]);
            f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < KS; ++y) {
                uint32_t f[4];
                f[0] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kw[u][y], s, 0));
                f[1] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kw[u][y], s, 1));
                f[2] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kw[u][y], s, 2));
                f[3] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kw[u][y], s, 3));
                const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{f[0], f[1], f[2], f[3]});
#pragma unroll
                for (int t = QT - 1; t >= 0; --t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[y][t], acc, 0, 0, 0);
            }
            st[u] = acc;
        }
        // running maximum (base 2), probabilities
        float x8[8], most = kNoKey;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float v = st[u][x] * c;
                x8[4 * u + x] = (sees >> (4 * u + x)) & 1 ? v : -INFINITY;
                most = fmaxf(most, x8[4 * u + x]);
            }
        most = fmaxf(most, __shfl_xor(most, 16, kWave));
        most = fmaxf(most, __shfl_xor(most, 32, kWave));
        const float m2 = fmaxf(m, most), a = fast_exp2(m - m2);
        m = m2;
        l *= a;
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] *= a;
        uint32_t pw[PT][4];
#pragma unroll
        for (int x = 0; x < 8; x += 2) {
            const float p0 = fast_exp2(x8[x] - m), p1 = fast_exp2(x8[x + 1] - m);
            l += p0 + p1;
            uint32_t a0[PT], a1[PT];
            split_bf16<PT>(p0, a0);
            split_bf16<PT>(p1, a1);
#pragma unroll
            for (int t = 0; t < PT; ++t) pw[t][x / 2] = a0[t] | (a1[t] << 16);
        }
        bf16x8 pf[PT];
#pragma unroll
        for (int t = 0; t < PT; ++t) pf[t] = __builtin_bit_cast(bf16x8, u32x4{pw[t][0], pw[t][1], pw[t][2], pw[t][3]});
        // V^T P^T: byte y of a token's share is channels 2 y and 2 y + 1 of this lane
#pragma unroll
        for (int y = 0; y < J / 2; ++y) {
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t w[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int at = t * (D / 32) + y;  // byte of the lane's load
                    const float s = scale_of((vsc[u] >> (8 * t)) & 0xFF);
                    const uint32_t src = vw[u][at / 4] >> (8 * (at % 4));
                    w[t] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(src, s, 0));
                }
                lo[2 * u] = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u);
                lo[2 * u + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u);
                hi[2 * u] = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
                hi[2 * u + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
            }
            const bf16x8 vl = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], lo[2], lo[3]});
            const bf16x8 vh = __builtin_bit_cast(bf16x8, u32x4{hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
            for (int t = PT - 1; t >= 0; --t) {
                o[2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vl, pf[t], o[2 * y], 0, 0, 0);
                o[2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, pf[t], o[2 * y + 1], 0, 0, 0);
            }
        }
    }

    // the waves' sums: rows of 16 queries, channel d/4 * b + d/16 * (register) + tile
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (lb == 0) { s_m[wv][n] = m; s_l[wv][n] = l; }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int j = 0; j < J; ++j) s_o[wv][n][lb * (D / 4) + x * J + j] = o[j][x];
    __syncthreads();
    const int rr = threadIdx.x >> 4, part = threadIdx.x & 15, r2 = r0 + rr;
    if (r2 >= live) return;
    float top = kNoKey, sum = 0.f, acc[J] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, s_m[w][rr]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float a = fast_exp2(s_m[w][rr] - top);
        sum = fmaf(s_l[w][rr], a, sum);
#pragma unroll
        for (int j = 0; j < J; ++j) acc[j] = fmaf(s_o[w][rr][part * J + j], a, acc[j]);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // a row that sees no key: zeros
    const int i2 = r2 / dim.G, h2 = h * dim.G + (r2 - i2 * dim.G);
    const long to = (long)b * o_lay.batch + (long)i2 * o_lay.token + (long)h2 * o_lay.head + part * J;
    if (F32) {
#pragma unroll
        for (int j = 0; j < J; ++j) static_cast<float*>(out)[to + j] = acc[j] * inv;
    } else {
#pragma unroll
        for (int j = 0; j < J; j += 2)
            *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(out) + to + j) = f32_to_bf16(acc[j] * inv) | (f32_to_bf16(acc[j + 1] * inv) << 16);
    }
    if (lse && part == 0)
        lse[((long)b * p.H * dim.G + h2) * dim.N + i2] = sum == 0.f ? -INFINITY : (top + fast_log2(sum)) * kLn2C;
}

// ------------------------------------------------------------------------------------------------ host

// What all calls share: the pool's shape.
int check_pool(const char* who, int H, int d, int n_pages, int page, int max_pages, Pool* p) {
    if (H <= 0 || d <= 0 || n_pages <= 0 || page <= 0 || max_pages <= 0) return fail(MD_EINVAL, "%s: sizes must be positive", who);
    if (d != 64 && d != 128) return fail(MD_ESHAPE, "%s: d=%d is not supported (64 or 128)", who, d);
    if (page < 16 || page > 256 || (page & (page - 1))) return fail(MD_ESHAPE, "%s: page=%d must be a power of two from 16 to 256", who, page);
    if ((long)n_pages * page > 0x7FFFFFFFl) return fail(MD_ESHAPE, "%s: a pool of %d pages of %d tokens has more slots than 31 bits name", who, n_pages, page);
    if ((long)max_pages * page > 0x7FFFFFFFl / 2) return fail(MD_ESHAPE, "%s: %d pages of %d tokens are too many for one request", who, max_pages, page);
    if (H > 65535) return fail(MD_ESHAPE, "%s: H=%d out of range", who, H);
    *p = Pool{n_pages, page, __builtin_ctz((unsigned)page), max_pages, H, (long)c4_page_bytes(page, d)};
    return MD_OK;
}
size_t pool_bytes(const Pool& p) { return (size_t)p.n_pages * p.H * p.stride; }

int check_dtype(const char* who, int dtype) {
    return dtype == MD_F32 || dtype == MD_BF16 ? MD_OK : fail(MD_EDTYPE, "%s: unknown dtype %d", who, dtype);
}

constexpr long kMaxGrid = 0x7FFFFFFFl;

struct Range { const void* p; size_t n; };
// None of the first `outs` ranges may share a byte with any other range.
int check_apart(const char* who, const Range* r, int outs, int all) {
    for (int a = 0; a < outs; ++a)
        for (int c = a + 1; c < all; ++c)
            if (overlaps(r[a].p, r[a].n, r[c].p, r[c].n)) return fail(MD_EALIAS, "%s: the outputs, the workspace and the inputs must not overlap", who);
    return MD_OK;
}

int pages_impl(const int32_t* new_len, int32_t* len, int32_t* table, int32_t* free_pages, int32_t* n_free, int32_t* slots, int32_t* missing,
               int B, int max_pages, int n_pages, int page, int N, void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    Pool p;
    int rc = check_pool("cache4_pages", 1, 64, n_pages, page, max_pages, &p);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N < 0) return fail(MD_EINVAL, "cache4_pages: B must be positive and N not negative");
    if (B > 65535) return fail(MD_ESHAPE, "cache4_pages: B=%d out of range", B);
    if ((long)B * max_pages > 0x7FFFFFFFl) return fail(MD_ESHAPE, "cache4_pages: a table of %d x %d entries is too large", B, max_pages);
    if (!new_len || !len || !table || !free_pages || !n_free || !missing || (N > 0 && !slots))
        return fail(MD_EINVAL, "cache4_pages: null pointer among the required arguments");
    if (!slots) N = 0;
    const size_t need = round_up((size_t)B * sizeof(PagePlan), 256);
    const Range r[] = {{len, (size_t)B * 4}, {table, (size_t)B * max_pages * 4}, {free_pages, (size_t)n_pages * 4}, {n_free, 4},
                       {slots, (size_t)B * N * 4}, {missing, 4}, {workspace, workspace ? need : 0}, {new_len, (size_t)B * 4}};
    rc = check_apart("cache4_pages", r, 7, 8);
    if (rc != MD_OK) return rc;
    if (!workspace || workspace_bytes < need)
        return fail(MD_EWORKSPACE, "cache4_pages: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(MD_EALIGN, "cache4_pages: workspace must be 256-byte aligned");
    PagePlan* plan = static_cast<PagePlan*>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    MD_LAUNCH("cache4_pages", st, (cache4_pages_kernel), 1, 1024, 0,
        new_len, len, table, free_pages, n_free, missing, B, max_pages, n_pages, p.page_shift, plan);
    const int most = N > max_pages ? N : max_pages;
    MD_LAUNCH("cache4_slots", st, (cache4_slots_kernel), dim3((most + 255) / 256, B), 256, 0,
        plan, table, free_pages, slots, max_pages, n_pages, p.page_shift, N);
    return check_launch("cache4_pages");
}

size_t rows_bytes(const KvLayout& l, int B, int N, int H, int d, int dtype) { return layout_extent_bytes(l, B, N, H, d) / 2 * elt_size(dtype); }

int write_impl(const void* k_new, const void* v_new, int dtype, const int32_t* slots, void* cache,
               int B, int N, int H, int d, int n_pages, int page, const md_kv_layout* rows_layout, void* stream)
{
    clear_error();
    Pool p;
    int rc = check_pool("cache4_write", H, d, n_pages, page, 1, &p);
    if (rc == MD_OK) rc = check_dtype("cache4_write", dtype);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N <= 0) return fail(MD_EINVAL, "cache4_write: sizes must be positive");
    if (!k_new || !v_new || !slots || !cache) return fail(MD_EINVAL, "cache4_write: null pointer among the required arguments");
    KvLayout lay;
    rc = read_layout("cache4_write", "rows", rows_layout, B, N, H, d, &lay);
    if (rc != MD_OK) return rc;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(cache)) return fail(MD_EALIGN, "cache4_write: tensors must be 16-byte aligned");
    const long rows = (long)B * N, blocks = ((rows + 3) / 4 * H + 3) / 4;
    if (blocks > kMaxGrid) return fail(MD_ESHAPE, "cache4_write: too many rows");
    const size_t in = rows_bytes(lay, B, N, H, d, dtype);
    const Range r[] = {{cache, pool_bytes(p)}, {k_new, in}, {v_new, in}, {slots, (size_t)rows * 4}};
    rc = check_apart("cache4_write", r, 1, 4);
    if (rc != MD_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_WRITE(D_, F_) MD_LAUNCH("cache4_write", st, (cache4_write_kernel<D_, F_>), (int)blocks, 256, 0, k_new, v_new, slots, static_cast<uint8_t*>(cache), p, lay, rows, N)
    if (d == 128) { if (dtype == MD_F32) MD_C4_WRITE(128, true); else MD_C4_WRITE(128, false); }
    else { if (dtype == MD_F32) MD_C4_WRITE(64, true); else MD_C4_WRITE(64, false); }
#undef MD_C4_WRITE
    return check_launch("cache4_write");
}

int read_impl(const void* cache, const int32_t* table, const int32_t* len, const int32_t* first, void* k_out, void* v_out, int dtype,
              int B, int N, int H, int d, int n_pages, int page, int max_pages, const md_kv_layout* rows_layout, void* stream)
{
    clear_error();
    Pool p;
    int rc = check_pool("cache4_read", H, d, n_pages, page, max_pages, &p);
    if (rc == MD_OK) rc = check_dtype("cache4_read", dtype);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N <= 0) return fail(MD_EINVAL, "cache4_read: sizes must be positive");
    if (!cache || !table || !len || !k_out || !v_out) return fail(MD_EINVAL, "cache4_read: null pointer among the required arguments");
    KvLayout lay;
    rc = read_layout("cache4_read", "rows", rows_layout, B, N, H, d, &lay);
    if (rc != MD_OK) return rc;
    if (!aligned16(k_out) || !aligned16(v_out) || !aligned16(cache)) return fail(MD_EALIGN, "cache4_read: tensors must be 16-byte aligned");
    const long rows = (long)B * N, blocks = ((rows + 3) / 4 * H + 3) / 4;
    if (blocks > kMaxGrid) return fail(MD_ESHAPE, "cache4_read: too many rows");
    const size_t outb = rows_bytes(lay, B, N, H, d, dtype);
    const Range r[] = {{k_out, outb}, {v_out, outb}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {first, first ? (size_t)B * 4 : 0}};
    rc = check_apart("cache4_read", r, 2, 6);
    if (rc != MD_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_READ(D_, F_) MD_LAUNCH("cache4_read", st, (cache4_read_kernel<D_, F_>), (int)blocks, 256, 0, static_cast<const uint8_t*>(cache), table, len, first, k_out, v_out, p, lay, rows, N)
    if (d == 128) { if (dtype == MD_F32) MD_C4_READ(128, true); else MD_C4_READ(128, false); }
    else { if (dtype == MD_F32) MD_C4_READ(64, true); else MD_C4_READ(64, false); }
#undef MD_C4_READ
    return check_launch("cache4_read");
}

size_t attend_bytes(int B, int N, int Hq, int H, int d, int max_pages, int page) {
    Pool p;
    if (B <= 0 || N <= 0 || Hq <= 0 || H <= 0 || Hq % H || check_pool("cache4_attend", H, d, 1, page, max_pages, &p) != MD_OK) return 0;
    return 256;
}

int attend_impl(const void* q, int dtype, const void* cache, const int32_t* table, const int32_t* len, const int32_t* q_len, const uint8_t* keep,
                int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, float softmax_scale,
                void* out, float* lse, const md_kv_layout* q_layout, const md_kv_layout* out_layout,
                void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    Pool p;
    int rc = check_pool("cache4_attend", H, d, n_pages, page, max_pages, &p);
    if (rc == MD_OK) rc = check_dtype("cache4_attend", dtype);
    if (rc != MD_OK) return rc;
    if (B <= 0 || N <= 0 || Hq <= 0) return fail(MD_EINVAL, "cache4_attend: sizes must be positive");
    if (Hq % H || Hq > 65535) return fail(MD_ESHAPE, "cache4_attend: Hq=%d must be a multiple of H=%d", Hq, H);
    if (!q || !cache || !table || !len || !out) return fail(MD_EINVAL, "cache4_attend: null pointer among the required arguments");
    if (!(softmax_scale > 0.f) || std::isinf(softmax_scale)) return fail(MD_EINVAL, "cache4_attend: softmax_scale must be positive and finite");
    KvLayout ql, ol;
    rc = read_layout("cache4_attend", "q", q_layout, B, N, Hq, d, &ql);
    if (rc == MD_OK) rc = read_layout("cache4_attend", "out", out_layout, B, N, Hq, d, &ol);
    if (rc != MD_OK) return rc;
    if (!aligned16(q) || !aligned16(out) || !aligned16(cache) || (reinterpret_cast<uintptr_t>(keep) & 3u))
        return fail(MD_EALIGN, "cache4_attend: tensors must be 16-byte aligned, keep 4-byte aligned");
    const int G = Hq / H;
    if ((long)N * G > 0x7FFFFFFFl - 64) return fail(MD_ESHAPE, "cache4_attend: too many query rows");
    const int tiles = (N * G + 15) / 16;
    const long blocks = (long)B * H * tiles;
    if (blocks > kMaxGrid) return fail(MD_ESHAPE, "cache4_attend: too many query rows");
    const size_t need = attend_bytes(B, N, Hq, H, d, max_pages, page);
    const Range r[] = {{out, rows_bytes(ol, B, N, Hq, d, dtype)}, {lse, lse ? (size_t)B * Hq * N * 4 : 0}, {workspace, workspace ? need : 0},
                       {q, rows_bytes(ql, B, N, Hq, d, dtype)}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {q_len, q_len ? (size_t)B * 4 : 0}, {keep, keep ? (size_t)B * max_pages * page : 0}};
    rc = check_apart("cache4_attend", r, 3, 9);
    if (rc != MD_OK) return rc;
    if (!workspace || workspace_bytes < need)
        return fail(MD_EWORKSPACE, "cache4_attend: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(MD_EALIGN, "cache4_attend: workspace must be 256-byte aligned");
    const AttendDims dim{B, N, G, tiles};
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_ATTEND(D_, F_) MD_LAUNCH("cache4_attend", st, (cache4_attend_kernel<D_, F_>), (int)blocks, 256, 0, \
        q, static_cast<const uint8_t*>(cache), table, len, q_len, keep, p, dim, softmax_scale, out, lse, ql, ol)
    if (d == 128) { if (dtype == MD_F32) MD_C4_ATTEND(128, true); else MD_C4_ATTEND(128, false); }
    else { if (dtype == MD_F32) MD_C4_ATTEND(64, true); else MD_C4_ATTEND(64, false); }
#undef MD_C4_ATTEND
    return check_launch("cache4_attend");
}

}  // namespace
}  // namespace md

extern "C" size_t mustdrop_cache4_bytes(int n_pages, int page, int H, int d)
{
    md::Pool p;
    md::clear_error();
    return md::check_pool("cache4_bytes", H, d, n_pages, page, 1, &p) == MD_OK ? md::pool_bytes(p) : 0;
}

extern "C" size_t mustdrop_cache4_pages_workspace_bytes(int B)
{
    return B > 0 ? md::round_up((size_t)B * sizeof(md::PagePlan), 256) : 0;
}

extern "C" size_t mustdrop_cache4_attend_workspace_bytes(int B, int N, int Hq, int H, int d, int max_pages, int page)
{
    md::clear_error();
    return md::attend_bytes(B, N, Hq, H, d, max_pages, page);
}

extern "C" int mustdrop_cache4_pages(
    const int32_t* new_len, int32_t* len, int32_t* table, int32_t* free_pages, int32_t* n_free, int32_t* slots, int32_t* missing,
    int B, int max_pages, int n_pages, int page, int N, void* workspace, size_t workspace_bytes, void* stream)
{
    return md::pages_impl(new_len, len, table, free_pages, n_free, slots, missing, B, max_pages, n_pages, page, N, workspace, workspace_bytes, stream);
}

extern "C" int mustdrop_cache4_write(
    const void* k_new, const void* v_new, md_dtype dtype, const int32_t* slots, void* cache,
    int B, int N, int H, int d, int n_pages, int page, const md_kv_layout* rows_layout, void* stream)
{
    return md::write_impl(k_new, v_new, dtype, slots, cache, B, N, H, d, n_pages, page, rows_layout, stream);
}

extern "C" int mustdrop_cache4_read(
    const void* cache, const int32_t* table, const int32_t* len, const int32_t* first, void* k_out, void* v_out, md_dtype dtype,
    int B, int N, int H, int d, int n_pages, int page, int max_pages, const md_kv_layout* rows_layout, void* stream)
{
    return md::read_impl(cache, table, len, first, k_out, v_out, dtype, B, N, H, d, n_pages, page, max_pages, rows_layout, stream);
}

extern "C" int mustdrop_cache4_attend(
    const void* q, md_dtype dtype, const void* cache, const int32_t* table, const int32_t* len, const int32_t* q_len, const uint8_t* keep,
    int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, float softmax_scale,
    void* out, float* lse, const md_kv_layout* q_layout, const md_kv_layout* out_layout,
    void* workspace, size_t workspace_bytes, void* stream)
{
    return md::attend_impl(q, dtype, cache, table, len, q_len, keep, B, N, Hq, H, d, n_pages, page, max_pages, softmax_scale,
                           out, lse, q_layout, out_layout, workspace, workspace_bytes, stream);
}
