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
//   cache4_attend_kernel                       softmax(scale Q K^T) V over the pages, a block per tile of query rows
//   cache4_attend_runs_kernel, cache4_join_*   the same in runs of equal work, whose parts are added up behind
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

// One sample's part of a call, handed on to whoever writes its entries and slots: lengths before and after, and the place on the
// stack of the first page that it takes.
struct PagePlan { int old_len, new_len, first; };

// Of 1024 samples whose entries follow one another from before[b] on, the one that entry x belongs to.
__device__ __forceinline__ int owner_of(const int* before, int x) {
    int b = 0;
#pragma unroll
    for (int step = 512; step; step >>= 1)
        if (before[b + step] <= x) b += step;
    return b;
}

__device__ __forceinline__ void write_slot(const PagePlan& p, int i, const int32_t* row, const int32_t* free_pages, int n_pages, int page_shift, int32_t* slot) {
    int s = -1;
    if (i < p.new_len - p.old_len) {
        const int at = p.old_len + i;
        const int e = at >> page_shift, held = c4_pages_of(p.old_len, page_shift), j = p.first - (e - held);
        const int id = c4_page_id(e < held ? row[e] : (j >= 0 && j < n_pages ? free_pages[j] : -1), n_pages);
        if (id >= 0) s = (int)(((uint32_t)id << page_shift) + (at & ((1 << page_shift) - 1)));
    }
    *slot = s;
}

// One block: counts the pages that leave and come, gives each sample its place on the stack and puts the released pages there.  The
// entries of 1024 samples are shared out evenly, four loads of a thread on their way together, whoever's they are.  ALL: the block takes the
// new pages and writes the slots too.
template <bool ALL>
__global__ __launch_bounds__(1024) void cache4_pages_kernel(
    const int32_t* __restrict__ new_len, int32_t* __restrict__ len, int32_t* table,
    int32_t* free_pages, int32_t* __restrict__ n_free, int32_t* __restrict__ slots, int32_t* __restrict__ missing,
    int B, int max_pages, int n_pages, int page_shift, int N, PagePlan* __restrict__ plan)
{
    __shared__ int s_red[16], s_before[1024];
    __shared__ PagePlan s_plan[1024];
    const int tid = threadIdx.x, top = c4_clamp(n_free[0], 0, n_pages);
    int leave = 0, come = 0;                         // (the host checks that B * max_pages + n_pages fits 31 bits)
    for (int b = tid; b < B; b += 1024) {
        const C4Change c = c4_change(len[b], new_len[b], max_pages, page_shift);
        if (c.held > c.need) leave += c.held - c.need;
        else come += c.need - c.held;
    }
    const int R = block_sum_i(leave, s_red), T = block_sum_i(come, s_red);
    const int left = top + R - T;
    if (tid == 0) {
        missing[0] = left < 0 ? -left : 0;
        if (left >= 0) n_free[0] = min(left, n_pages);
    }
    int left_before = 0, come_before = 0;
    for (int b0 = 0; b0 < B; b0 += 1024) {
        const int b = b0 + tid;
        C4Change c{0, 0, 0, 0};
        if (b < B && left >= 0) c = c4_change(len[b], new_len[b], max_pages, page_shift);
        int lt, ct;
        const int lp = block_exscan_i(max(c.held - c.need, 0), s_red, lt), cp = block_exscan_i(max(c.need - c.held, 0), s_red, ct);
        const PagePlan mine{c.old_len, c.new_len, c4_taken_at(top, R, come_before + cp)};
        s_plan[tid] = mine;
        s_before[tid] = lp;
        if (b < B) {
            if (left >= 0) len[b] = c.new_len;
            if (!ALL) plan[b] = mine;
        }
        __syncthreads();
        for (int x0 = tid; x0 < lt; x0 += 4096) {
            int id[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = x0 + i * 1024;
                if (x >= lt) continue;
                const int from = owner_of(s_before, x);
                id[i] = table[(long)(b0 + from) * max_pages + c4_pages_of(s_plan[from].new_len, page_shift) + x - s_before[from]];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = x0 + i * 1024, at = c4_released_at(top, R, left_before + x);
                if (x < lt && at < n_pages) free_pages[at] = id[i];
            }
        }
        left_before += lt;
        come_before += ct;
        __syncthreads();
        if (!ALL) continue;
        s_before[tid] = cp;                          // (ALL has one round: every page that is taken is on the stack by now)
        __syncthreads();
        for (int x0 = tid; x0 < ct; x0 += 4096) {
            int id[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = c4_taken_at(top, R, x0 + i * 1024);
                id[i] = x0 + i * 1024 < ct && at < n_pages ? free_pages[at] : -1;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = x0 + i * 1024;
                if (x >= ct || c4_taken_at(top, R, x) >= n_pages) continue;
                const int to = owner_of(s_before, x);
                table[(long)to * max_pages + c4_pages_of(s_plan[to].old_len, page_shift) + x - s_before[to]] = id[i];
            }
        }
    }
    if (ALL)
        for (int x = tid; x < B * N; x += 1024) {
            const int b = x / N;
            write_slot(s_plan[b], x - b * N, table + (long)b * max_pages, free_pages, n_pages, page_shift, slots + x);
        }
}

// Entries and slots of one sample per blockIdx.y.
__global__ __launch_bounds__(256) void cache4_slots_kernel(
    const PagePlan* __restrict__ plan, int32_t* __restrict__ table, const int32_t* __restrict__ free_pages,
    int32_t* __restrict__ slots, int max_pages, int n_pages, int page_shift, int N)
{
    const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    const PagePlan p = plan[b];
    const int held = c4_pages_of(p.old_len, page_shift), need = c4_pages_of(p.new_len, page_shift);
    int32_t* row = table + (long)b * max_pages;
    // place `first - j` of the stack holds the j-th page that the sample takes
    if (i < need - held && p.first - i >= 0 && p.first - i < n_pages) row[held + i] = free_pages[p.first - i];
    if (slots && i < N) write_slot(p, i, row, free_pages, n_pages, page_shift, slots + (long)b * N + i);
}

// ------------------------------------------------------------------------------------------------ rows in and out

// Heads that a wave of the copies takes: one, unless there are waves for all of the chip more than once; then two on the way in and
// four on the way out.  us with one / two / four heads: 16 x up to 640 rows of 32 heads in 30.5 / 29.3 / 28.4, out 27.1 / 25.2 / 23.9; 4 x 777
// fp32 rows of 40 heads of 64 in 13.2 / 13.1 / 13.9; 64 x 1025 rows out 369 / 313 / 295; 64 rows in 3.0 / 3.8 / 4.4, 4 x 160 rows of 40 heads out 4.4 /
// 4.6 / 4.8.  Rows out by streaming stores: 64 x 1025 rows 318 us with plain ones, 4 x 160 rows 5.3, and what follows does not wait for their
// lines to leave the caches (rows in behind rows out 28.4 us, 36.7 behind plain stores).
constexpr long kManyWaves = 16384;
inline bool many_rows(long rows, int H) { return (rows + 3) / 4 * H >= kManyWaves; }

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

// A wave writes four rows, sixteen lanes per row with d/16 channels each, of HEADS heads: their loads are on their way together.
template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void cache4_write_kernel(
    const void* __restrict__ k_new, const void* __restrict__ v_new, const int32_t* __restrict__ slots, uint8_t* __restrict__ cache,
    Pool p, KvLayout lay, int rows, int N)
{
    const int lane = lane_id(), part = lane & 15, h0 = blockIdx.y * HEADS;
    const int r = (int)blockIdx.x * 16 + wave_id() * 4 + (lane >> 4);        // (the host checks that this fits 31 bits)
    C4Slot at{-1, 0};
    if (r < rows) at = c4_slot(slots[r], p.n_pages, p.page_shift);
    float k[HEADS][D / 16] = {}, v[HEADS][D / 16] = {};
    if (at.page >= 0) {
        const int b = r / N;
        const long from = b * lay.batch + (long)(r - b * N) * lay.token + part * (D / 16);
#pragma unroll
        for (int x = 0; x < HEADS; ++x)
            if (h0 + x < p.H) {
                load_part<D, F32>(k_new, from + (long)(h0 + x) * lay.head, k[x]);
                load_part<D, F32>(v_new, from + (long)(h0 + x) * lay.head, v[x]);
            }
    }
    const int group = part / (512 / D);
    uint8_t* to = cache + ((long)at.page * p.H + h0) * p.stride;
#pragma unroll
    for (int x = 0; x < HEADS; ++x) {
        int ks, vs;
        const uint32_t kw = quantise_part<D>(k[x], ks), vw = quantise_part<D>(v[x], vs);
        if (at.page < 0 || h0 + x >= p.H) continue;
        store_codes<D>(to + c4_k_codes(at.place, D) + part * (D / 32), kw);
        store_codes<D>(to + c4_v_codes(p.page, at.place, part, D), vw);
        if (part % (512 / D) == 0) {
            to[c4_k_scales(p.page, at.place, D) + group] = (uint8_t)ks;
            to[c4_v_scales(p.page, at.place, group, D)] = (uint8_t)vs;
        }
        to += p.stride;
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
        f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(base) + at);
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
        __builtin_nontemporal_store(f32x4{a.x, a.y, b.x, b.y}, p);
        if (D == 128) {
            const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
            __builtin_nontemporal_store(f32x4{c.x, c.y, d.x, d.y}, p + 1);
        }
    } else {
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        const uint32_t a = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)), b = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        if (D == 128) {
            const u32x4 v{a, b, as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)), as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
        } else {
            __builtin_nontemporal_store(u32x2{a, b}, reinterpret_cast<u32x2*>(p));
        }
    }
}

// The way back, shared out as in the write.
template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void cache4_read_kernel(
    const uint8_t* __restrict__ cache, const int32_t* __restrict__ table, const int32_t* __restrict__ len, const int32_t* __restrict__ first,
    void* __restrict__ k_out, void* __restrict__ v_out, Pool p, KvLayout lay, int rows, int N)
{
    const int lane = lane_id(), part = lane & 15, h0 = blockIdx.y * HEADS;
    const int r = (int)blockIdx.x * 16 + wave_id() * 4 + (lane >> 4);
    if (r >= rows) return;
    const int b = r / N, i = r - b * N;
    const long at = (first ? (long)first[b] : 0l) + i;
    if (at < 0 || at >= c4_clamp(len[b], 0, p.max_pages << p.page_shift)) return;
    const int t = (int)at & (p.page - 1), id = c4_page_id(table[(long)b * p.max_pages + ((int)at >> p.page_shift)], p.n_pages);
    if (id < 0) return;
    const uint8_t* from = cache + ((long)id * p.H + h0) * p.stride;
    const int group = part / (512 / D);
    uint32_t kw[HEADS], vw[HEADS], ks[HEADS], vs[HEADS];
#pragma unroll
    for (int x = 0; x < HEADS; ++x)
        if (h0 + x < p.H) {
            kw[x] = load_codes<D>(from + c4_k_codes(t, D) + part * (D / 32));
            vw[x] = load_codes<D>(from + c4_v_codes(p.page, t, part, D));
            ks[x] = from[c4_k_scales(p.page, t, D) + group];
            vs[x] = from[c4_v_scales(p.page, t, group, D)];
            from += p.stride;
        }
    const long to = b * lay.batch + i * lay.token + part * (D / 16);
#pragma unroll
    for (int x = 0; x < HEADS; ++x)
        if (h0 + x < p.H) {
            store_values<D, F32>(k_out, to + (long)(h0 + x) * lay.head, kw[x], ks[x]);
            store_values<D, F32>(v_out, to + (long)(h0 + x) * lay.head, vw[x], vs[x]);
        }
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
    int end, clear;                                  // keys that any row sees; that all rows see and no mask may leave out
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
    w.clear = A.keep ? 0 : min(max(s.length - s.nq + first_row / A.dim.G + 1, 0), w.end);
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
__device__ __forceinline__ Early early_pages(const Walk& w, int first, int stride) {
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

    // Keys of the step that the call leaves out for all rows get a V scale of 1 (0 * NaN would count); `hides` gets a bit for each
    // of the lane's eight keys that its row does not see: of key x of tile u bit 8 x + 7 - 4 u.  Four keys at a time, a byte each.
    __device__ __forceinline__ void mask(const Walk& w, int step, const Kept& kp, uint32_t (&vs)[2], uint32_t (&hides)[NT]) {
        constexpr uint32_t kTops = 0x80808080u;
        const auto nonzero = [](uint32_t x) { return (((x & ~kTops) + ~kTops) | x) & kTops; };
        const auto first = [](int n) { return n <= 0 ? 0u : kTops >> (32 - 8 * min(n, 4)); };
        const Pages pg = pages_at(w, step);
        const bool ok[2] = {there(w, step, pg, 0), there(w, step, pg, 1)};
        uint32_t nan = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) hides[t] = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = step * 32 + 16 * u + 4 * lb;
            const uint32_t w0 = kp.w[u][0], w1 = kp.w[u][1], w2 = kp.w[u][2], w3 = kp.w[u][3];
            const uint32_t even = lb & 2 ? w2 : w0, odd = lb & 2 ? w3 : w1, kept = lb & 1 ? odd : even;
            const uint32_t on = nonzero(kept) & first((ok[u] ? w.end : 0) - t), nans = kTops & ~nonzero(~vs[u]);
            nan |= on & nans;
#pragma unroll
            for (int z = 0; z < NT; ++z) hides[z] |= (on & first(limit[z] - t)) >> (4 * u);
            const uint32_t out = (kTops & ~on) | nans, bytes = (out << 1) - (out >> 7);
            vs[u] = (vs[u] & ~bytes) | (bytes & 0x7F7F7F7Fu);
        }
#pragma unroll
        for (int z = 0; z < NT; ++z) hides[z] = ~hides[z];
        // A NaN in V of a key that some rows see and others do not: the rows that see it get it in that group's channels here.
        if (__any(nan != 0)) {
#pragma unroll
            for (int z = 0; z < NT; ++z) {
                float poison = 0.f;
#pragma unroll 1
                for (int x = 0; x < 32; ++x) {
                    const int t = step * 32 + x, id = x < 16 ? pg.id[0] : pg.id[1];
                    if (!(x < 16 ? ok[0] : ok[1]) || t >= w.end || (w.keep && ((w.keep[t >> 2] >> (8 * (t & 3))) & 0xFF) == 0)) continue;
                    if (t < limit[z] && page_base(w, id)[c4_v_scales(w.page, t & (w.page - 1), lb * D / 128, D)] == 255) poison = __builtin_nanf("");
                }
#pragma unroll
                for (int j = 0; j < J; ++j) o[z][j] += poison;
            }
        }
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

    __device__ __forceinline__ void step(const Walk& w, const Keys& K, bool masked, uint32_t (&hides)[NT]) {
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
    __device__ __forceinline__ void run(const Walk& w, int first, int stop, int stride, char* ring, const Early& early) {
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
            const bool masked = ((holes >> x) & 1) != 0 || i * 32 + 32 > w.clear;
            holes &= ~(1u << x);
            if (ahead < stop) {
                if (hole(w, ahead, pg)) holes |= 1u << x;
                ask(w, ahead, pg, ring + x * SLOT);
            }
            x = x + 1 == RING ? 0 : x + 1;
            uint32_t hides[NT];
            if (masked) R::mask(w, i, kp, k.vs, hides);
            step(w, k, masked, hides);
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

// The sample of the blocks that come `at`-th: of each 64, the longest first, so that the last blocks to run are short.  us as they come / so, of
// 32 heads on 8: a prompt's piece of 4 x 512 tokens behind up to 5888 keys 257 / 235, 32 x 128 behind up to 4000 318 / 300.  It gains nothing
// where lengths are equal or the blocks make many rounds anyway, and then costs what the order takes to find: 8 x 512 behind 1500 keys each
// 177 / 183, 16 x 512 behind up to 3000 389 / 405, 64 x 512 behind up to 1500 845 / 950.  Not for single tokens, which wait for memory: 64 x
// up to 4096 keys 114 / 122, 64 x up to 500 26 / 33.
__device__ __forceinline__ int by_length(const AttendArgs& A, int at) {
    const int base = at & -kWave, lane = lane_id(), n = min(A.dim.B - base, kWave);
    int mine = -1, before = 0;
    if (lane < n) {
        mine = c4_clamp(global(A.len)[base + lane], 0, A.p.max_pages << A.p.page_shift);
        if (A.q_len && global(A.q_len)[base + lane] <= 0) mine = 0;
    }
    for (int j = 0; j < n; ++j) {
        const int other = __builtin_amdgcn_readlane(mine, j);
        before += other > mine || (other == mine && j < lane) ? 1 : 0;
    }
    return base + (int)__builtin_ctzll(__ballot(lane < n && before == at - base));
}

// A block per tile of query rows of a (sample, K/V head); its waves take the steps in turn.
template <int D, bool F32, int NT, bool STREAM>
__global__ __launch_bounds__(NT == 2 || (F32 && D == 128) ? 256 : 512, NT == 2 || (F32 && D == 128) ? 3 : 4) void cache4_attend_kernel(AttendArgs A0)
{
    extern __shared__ f32x4 s_lds[];
    constexpr int ROWS = 16 * NT;
    Sweep<D, F32, NT, STREAM> sw;
    Walk w;
    Early early;
    int b;
    {
        const AttendArgs A = argument<AttendArgs>(0);
        const int tile = blockIdx.x % A.dim.tiles, bh = blockIdx.x / A.dim.tiles, h = bh % A.p.H, r0 = tile * ROWS;
        b = bh / A.p.H;
        if (NT == 2 && A.dim.B > 1) b = by_length(A, b);
        w = table_of(A, b);
        early = early_pages(w, wave_id(), blockDim.x >> 6);
        Sample s = sample_of(A, b);
        if (NT == 1) arrived(early, s.length, s.nq);             // (32 rows together are many steps to a wave: a prompt's piece 235 us either way)
        if (r0 >= s.nq * A.dim.G) return;
        sw.begin(A, s, h, r0);
        walk_of(w, A, s, h, r0, min(r0 + ROWS, s.nq * A.dim.G) - 1);
    }
    char* lds = reinterpret_cast<char*>(s_lds);
    sw.run(w, wave_id(), 0x7FFFFFFF, blockDim.x >> 6, lds + wave_id() * (sw.RING * sw.SLOT), early);
    __syncthreads();
    const AttendArgs A = argument<AttendArgs>(0);
    const int tile = blockIdx.x % A.dim.tiles, h = blockIdx.x / A.dim.tiles % A.p.H, r0 = tile * ROWS;
    const Sample s = sample_of(A, b);
    join_waves<D, NT>(sw, min(ROWS, s.nq * A.dim.G - r0), reinterpret_cast<float*>(s_lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
        store_out<D, F32>(A, b, h, r0 + row, part, x, m, l);
    });
}

// All samples' work, added up by a wave: the total, and where sample `b` begins or which sample holds the first step of a run.
struct Place { int total, b, begin; };
__device__ __forceinline__ Place find_place(const AttendArgs& A, int tile_rows, int b, bool by_run, int run, int blocks, int least) {
    const int cap = A.p.max_pages << A.p.page_shift, lane = lane_id();
    auto work_of = [&](int x) {
        if (x >= A.dim.B) return 0;
        const C4Work w = c4_work(c4_clamp(global(A.len)[x], 0, cap), (A.q_len ? c4_clamp(global(A.q_len)[x], 0, A.dim.N) : A.dim.N) * A.dim.G, tile_rows);
        return A.p.H * w.tiles * w.steps;
    };
    Place r{0, 0, 0};
    const int mine = work_of(lane), incl = wave_incl_scan_i(mine);       // of the first 64 samples, which are often all
    r.total = __builtin_amdgcn_readlane(incl, kWave - 1);
    for (int x = kWave; x < A.dim.B; x += kWave) r.total += wave_sum_i(work_of(x + lane));
    int at = 0;
    if (by_run) {
        const int runs = c4_runs(r.total, blocks, least);
        if (run >= runs || r.total == 0) { r.b = -1; return r; }
        at = c4_run_begin(run, r.total, runs);
    }
    int base = 0;
    for (int x = 0; x < A.dim.B; x += kWave) {
        const int w = x ? work_of(x + lane) : mine, in = x ? wave_incl_scan_i(w) : incl, sum = __builtin_amdgcn_readlane(in, kWave - 1);
        if (by_run ? at < base + sum : b < x + kWave) {
            const int l = by_run ? (int)__builtin_ctzll(__ballot(base + in > at)) : b - x;
            r.b = x + l;
            r.begin = base + __builtin_amdgcn_readlane(in, l) - __builtin_amdgcn_readlane(w, l);
            return r;
        }
        base += sum;
    }
    r.b = -1;
    return r;
}

// A block's run of steps, unit by unit: each(sample, K/V head, first row, first and last step, place of the part or -1).
template <class Each>
__device__ __forceinline__ void each_unit(int tile_rows, int run, Each each) {
    int at, stop, b, begin, total, runs;
    {
        const AttendArgs A = argument<AttendArgs>(0);
        const Parts parts = argument<Parts>(kPartsAt);
        const Place place = find_place(A, tile_rows, 0, true, run, parts.blocks, parts.least);
        if (place.b < 0) return;
        total = place.total;
        runs = c4_runs(total, parts.blocks, parts.least);
        at = c4_run_begin(run, total, runs);
        stop = c4_run_begin(run + 1, total, runs);
        b = place.b;
        begin = place.begin;
    }
    while (at < stop) {
        const AttendArgs A = argument<AttendArgs>(0);
        const Sample s = sample_of(A, b);
        const C4Work w = c4_work(s.length, s.nq * A.dim.G, tile_rows);
        const int whole = A.p.H * w.tiles * w.steps;
        if (at - begin >= whole) { begin += whole; ++b; continue; }
        const int unit = (at - begin) / w.steps, first = at - begin - unit * w.steps, last = min(w.steps, first + stop - at);
        const int h = unit / w.tiles, r0 = (unit - h * w.tiles) * tile_rows;
        each(A, s, h, r0, first, last, first == 0 && last == w.steps ? -1 : c4_part_place(run, begin + unit * w.steps, total, runs));
        at += last - first;
    }
}

// Few units, or units of unequal length: every block takes a run of as many steps, over the borders of units and samples.  A unit that
// lies within a run is finished there, the parts of the others are joined by the next kernel.
template <int D, bool F32, int NT, bool STREAM>
__global__ __launch_bounds__(256, NT == 2 || (F32 && D == 128) ? 3 : 4) void cache4_attend_runs_kernel(AttendArgs A0, Parts parts0)
{
    extern __shared__ f32x4 s_lds[];
    constexpr int ROWS = 16 * NT;
    char* lds = reinterpret_cast<char*>(s_lds);
    each_unit(ROWS, blockIdx.x, [&](const AttendArgs& A, const Sample& s, int h, int r0, int first, int last, int place) {
        Sweep<D, F32, NT, STREAM> sw;
        Walk w = table_of(A, s.b);
        const Early early = early_pages(w, first + wave_id(), 4);
        sw.begin(A, s, h, r0);
        const int rows = min(ROWS, s.nq * A.dim.G - r0), b = s.b;
        walk_of(w, A, s, h, r0, r0 + rows - 1);
        sw.run(w, first + wave_id(), last, 4, lds + wave_id() * (sw.RING * sw.SLOT), early);
        __syncthreads();
        const AttendArgs again = argument<AttendArgs>(0);
        const Parts parts = argument<Parts>(kPartsAt);
        join_waves<D, NT>(sw, rows, reinterpret_cast<float*>(s_lds), [&](int row, int part, const float (&x)[D / 16], float m, float l) {
            if (place < 0) store_out<D, F32>(again, b, h, r0 + row, part, x, m, l);
            else store_part<D>(parts, place, ROWS, row, part, x, m, l);
        });
        __syncthreads();
    });
}

// The parts of a unit that its runs left, and the runs that left them.
struct Cut { int begin, p0, p1, total, runs; };
__device__ __forceinline__ Cut cut_of(const AttendArgs& A, const Parts& parts, const Sample& s, int h, int tile, int tile_rows) {
    const Place place = find_place(A, tile_rows, s.b, false, 0, 0, 1);
    const C4Work w = c4_work(s.length, s.nq * A.dim.G, tile_rows);
    Cut c;
    c.total = place.total;
    c.runs = c4_runs(place.total, parts.blocks, parts.least);
    c.begin = place.begin + (h * w.tiles + tile) * w.steps;
    c.p0 = c4_run_of(c.begin, c.total, c.runs);
    c.p1 = c4_run_of(c.begin + w.steps - 1, c.total, c.runs);
    return c;
}
// One wave adds up parts x0, x0 + stride, .. of a row, 64 of them at a time: their weights side by side, their rows one after the other.
// A lane gets d/64 channels.
template <int D>
__device__ __forceinline__ void add_parts(const Parts& parts, const Cut& c, int x0, int stride, int row, int tile_rows, float& m, float& l, float (&acc)[D / 64]) {
    constexpr int C = D / 64;
    const int lane = lane_id();
    m = kNoKey;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) acc[j] = 0.f;
    for (; x0 <= c.p1; x0 += stride * kWave) {
        const int p = x0 + lane * stride;
        const bool on = p <= c.p1;
        const float2 ml = on ? parts.ml[(long)c4_part_place(p, c.begin, c.total, c.runs) * tile_rows + row] : float2{kNoKey, 0.f};
        const int n = min(kWave, (c.p1 - x0) / stride + 1);
        float v[8][C];
        const auto ask = [&](int y0) {
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const int q = x0 + min(y0 + y, n - 1) * stride;
                const float* from = parts.o + ((long)c4_part_place(q, c.begin, c.total, c.runs) * tile_rows + row) * D + lane * C;
#pragma unroll
                for (int j = 0; j < C; ++j) v[y][j] = from[j];
            }
        };
        ask(0);                                      // (on their way while the weights come and are worked out)
        const float top = fmaxf(m, wave_max(ml.x)), a = fast_exp2(m - top), e = on ? fast_exp2(ml.x - top) : 0.f;
        l = l * a + wave_sum(ml.y * e);
        m = top;
#pragma unroll
        for (int j = 0; j < C; ++j) acc[j] *= a;
        for (int y0 = 0; y0 < n; y0 += 8) {
            if (y0) ask(y0);
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const float f = y0 + y < n ? lane_bcast_f(e, y0 + y) : 0.f;
                if (y0 + y < n)
#pragma unroll
                    for (int j = 0; j < C; ++j) acc[j] = fmaf(v[y][j], f, acc[j]);
            }
        }
    }
}

// Few rows: a block per query row, its waves share the parts.
template <int D, bool F32>
__global__ __launch_bounds__(1024) void cache4_join_kernel(AttendArgs A, Parts parts, int tile_rows)
{
    __shared__ float s_o[16][D];
    __shared__ float s_m[16], s_l[16];
    const int rows = A.dim.N * A.dim.G, r = blockIdx.x % rows, bh = blockIdx.x / rows, h = bh % A.p.H, b = bh / A.p.H;
    const Sample s = sample_of(A, b);
    if (r >= s.nq * A.dim.G) return;
    const Cut c = cut_of(A, parts, s, h, r / tile_rows, tile_rows);
    if (c.p0 == c.p1) return;                        // finished in its run
    const int lane = lane_id(), wv = wave_id(), nw = blockDim.x >> 6;
    constexpr int C = D / 64;
    float m, l, acc[C];
    add_parts<D>(parts, c, c.p0 + wv, nw, r % tile_rows, tile_rows, m, l, acc);
#pragma unroll
    for (int j = 0; j < C; ++j) s_o[wv][lane * C + j] = acc[j];
    if (lane == 0) { s_m[wv] = m; s_l[wv] = l; }
    __syncthreads();
    if (threadIdx.x >= 16) return;
    const int part = threadIdx.x;
    float top = kNoKey, sum = 0.f, x[D / 16] = {};
    for (int y = 0; y < nw; ++y) top = fmaxf(top, s_m[y]);
    for (int y = 0; y < nw; ++y) {
        const float a = fast_exp2(s_m[y] - top);
        sum = fmaf(s_l[y], a, sum);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) x[j] = fmaf(s_o[y][part * (D / 16) + j], a, x[j]);
    }
    store_out<D, F32>(A, b, h, r, part, x, top, sum);
}

// Many rows, and then few parts of each: a block per sixteen rows of a unit, sixteen lanes per row.
template <int D, bool F32>
__global__ __launch_bounds__(256) void cache4_join_tiles_kernel(AttendArgs A, Parts parts, int tile_rows)
{
    const int groups = tile_rows / 16, group = blockIdx.x % groups, unit = blockIdx.x / groups;
    const int tile = unit % A.dim.tiles, bh = unit / A.dim.tiles, h = bh % A.p.H, b = bh / A.p.H;
    const Sample s = sample_of(A, b);
    const int row = group * 16 + (threadIdx.x >> 4), r = tile * tile_rows + row, part = threadIdx.x & 15, live = s.nq * A.dim.G;
    if (tile * tile_rows + group * 16 >= live) return;
    const Cut c = cut_of(A, parts, s, h, tile, tile_rows);
    if (c.p0 == c.p1 || r >= live) return;
    float m = kNoKey, l = 0.f, acc[D / 16] = {};
    for (int p0 = c.p0; p0 <= c.p1; p0 += 4) {
        float2 ml[4];
        f32x4 v[4][D / 64];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const long at = (long)c4_part_place(min(p0 + y, c.p1), c.begin, c.total, c.runs) * tile_rows + row;
            ml[y] = p0 + y <= c.p1 ? parts.ml[at] : float2{kNoKey, 0.f};
#pragma unroll
            for (int j = 0; j < D / 64; ++j) v[y][j] = reinterpret_cast<const f32x4*>(parts.o + at * D + part * (D / 16))[j];
        }
        const float top = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m), a = fast_exp2(m - top);
        m = top;
        l *= a;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) acc[j] *= a;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if (p0 + y > c.p1) break;
            const float e = fast_exp2(ml[y].x - top);
            l = fmaf(ml[y].y, e, l);
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc[j] = fmaf(v[y][j >> 2][j & 3], e, acc[j]);
        }
    }
    store_out<D, F32>(A, b, h, r, part, acc, m, l);
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
    if (B > 65535 || N > (1 << 30)) return fail(MD_ESHAPE, "cache4_pages: B=%d or N=%d out of range", B, N);
    // (places of the stack are counted in 31 bits, beyond its height by all that the tables could release, and the kernel looks 4096 ahead)
    if ((long)B * max_pages + n_pages > 0x7FFFFFFFl - 8192)
        return fail(MD_ESHAPE, "cache4_pages: a table of %d x %d entries and %d pages are too many", B, max_pages, n_pages);
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
    // One launch while a thread has up to 16 slots to write, else a second one with all of the chip.  us of a call that grows and one that
    // shrinks, one launch / two: 1 x 1 to 64 x 256 slots 14.5 / 18.3 (the host's time), 64 x 512 19.6 / 18.2, 256 x 128 19.7 / 18.0.
    if (B <= 1024 && (long)B * N <= 16384) {
        MD_LAUNCH("cache4_pages", st, (cache4_pages_kernel<true>), 1, 1024, 0,
            new_len, len, table, free_pages, n_free, slots, missing, B, max_pages, n_pages, p.page_shift, N, plan);
    } else {
        MD_LAUNCH("cache4_pages", st, (cache4_pages_kernel<false>), 1, 1024, 0,
            new_len, len, table, free_pages, n_free, slots, missing, B, max_pages, n_pages, p.page_shift, N, plan);
        const int most = N > max_pages ? N : max_pages;
        MD_LAUNCH("cache4_slots", st, (cache4_slots_kernel), dim3((most + 255) / 256, B), 256, 0,
            plan, table, free_pages, slots, max_pages, n_pages, p.page_shift, N);
    }
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
    const long rows = (long)B * N;
    if (rows > kMaxRows) return fail(MD_ESHAPE, "cache4_write: %ld rows are too many for one call", rows);
    const size_t in = rows_bytes(lay, B, N, H, d, dtype);
    const Range r[] = {{cache, pool_bytes(p)}, {k_new, in}, {v_new, in}, {slots, (size_t)rows * 4}};
    rc = check_apart("cache4_write", r, 1, 4);
    if (rc != MD_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_WRITE2(D_, F_, X_)                                                                                                          \
    MD_LAUNCH("cache4_write", st, (cache4_write_kernel<D_, F_, X_>), dim3((int)((rows + 15) / 16), (H + X_ - 1) / X_), 256, 0,            \
        k_new, v_new, slots, static_cast<uint8_t*>(cache), p, lay, (int)rows, N)
#define MD_C4_WRITE(D_, F_) do { if (many_rows(rows, H)) MD_C4_WRITE2(D_, F_, 2); else MD_C4_WRITE2(D_, F_, 1); } while (0)
    if (d == 128) { if (dtype == MD_F32) MD_C4_WRITE(128, true); else MD_C4_WRITE(128, false); }
    else { if (dtype == MD_F32) MD_C4_WRITE(64, true); else MD_C4_WRITE(64, false); }
#undef MD_C4_WRITE
#undef MD_C4_WRITE2
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
    const long rows = (long)B * N;
    if (rows > kMaxRows) return fail(MD_ESHAPE, "cache4_read: %ld rows are too many for one call", rows);
    const size_t outb = rows_bytes(lay, B, N, H, d, dtype);
    const Range r[] = {{k_out, outb}, {v_out, outb}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {first, first ? (size_t)B * 4 : 0}};
    rc = check_apart("cache4_read", r, 2, 6);
    if (rc != MD_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
#define MD_C4_READ2(D_, F_, X_)                                                                                                           \
    MD_LAUNCH("cache4_read", st, (cache4_read_kernel<D_, F_, X_>), dim3((int)((rows + 15) / 16), (H + X_ - 1) / X_), 256, 0,              \
        static_cast<const uint8_t*>(cache), table, len, first, k_out, v_out, p, lay, (int)rows, N)
#define MD_C4_READ(D_, F_) do { if (many_rows(rows, H)) MD_C4_READ2(D_, F_, 4); else MD_C4_READ2(D_, F_, 1); } while (0)
    if (d == 128) { if (dtype == MD_F32) MD_C4_READ(128, true); else MD_C4_READ(128, false); }
    else { if (dtype == MD_F32) MD_C4_READ(64, true); else MD_C4_READ(64, false); }
#undef MD_C4_READ
#undef MD_C4_READ2
    return check_launch("cache4_read");
}

struct AttendPlan {
    C4Attend cut;
    Parts parts;
    size_t lds, bytes;
};
AttendPlan attend_plan(void* workspace, bool f32, int B, int N, int Hq, int d, const Pool& p) {
    AttendPlan a;
    const int G = Hq / p.H, few = N * G < 16 ? N * G : 16;
    a.cut = c4_attend(f32, B, N, G, p.H, d, (int64_t)p.max_pages * p.page);
    const size_t join = sizeof(float) * ((size_t)a.cut.waves * few * (d + 4) + 2 * a.cut.waves * 16), ring = (size_t)a.cut.waves * kRing * (32 * d + 256);
    a.lds = join > ring ? join : ring;
    Carver c(workspace);
    const size_t places = a.cut.runs ? (size_t)2 * kC4Blocks * a.cut.tile_rows : 0;
    a.parts.o = c.take<float>(places * d);
    a.parts.ml = c.take<float2>(places);
    a.parts.blocks = kC4Blocks;
    a.parts.least = kC4Least;
    a.bytes = c.off > 256 ? c.off : 256;
    return a;
}

size_t attend_bytes(int B, int N, int Hq, int H, int d, int max_pages, int page) {
    Pool p;
    if (B <= 0 || N <= 0 || Hq <= 0 || H <= 0 || Hq % H || check_pool("cache4_attend", H, d, 1, page, max_pages, &p) != MD_OK) return 0;
    if ((long)N * (Hq / H) > 0x7FFFFFFFl - 128) return 0;
    const size_t x = attend_plan(nullptr, false, B, N, Hq, d, p).bytes, y = attend_plan(nullptr, true, B, N, Hq, d, p).bytes;
    return x > y ? x : y;
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
    // (the kernels take scores to base 2: an infinite factor would make a score of 0 no number)
    if (!(softmax_scale > 0.f) || std::isinf(softmax_scale * kLog2eC)) return fail(MD_EINVAL, "cache4_attend: softmax_scale must be positive and finite, times log2(e) too");
    KvLayout ql, ol;
    rc = read_layout("cache4_attend", "q", q_layout, B, N, Hq, d, &ql);
    if (rc == MD_OK) rc = read_layout("cache4_attend", "out", out_layout, B, N, Hq, d, &ol);
    if (rc != MD_OK) return rc;
    if (!aligned16(q) || !aligned16(out) || !aligned16(cache) || (reinterpret_cast<uintptr_t>(keep) & 3u))
        return fail(MD_EALIGN, "cache4_attend: tensors must be 16-byte aligned, keep 4-byte aligned");
    const int G = Hq / H;
    if ((long)N * G > 0x7FFFFFFFl - 128) return fail(MD_ESHAPE, "cache4_attend: too many query rows");
    const AttendPlan plan = attend_plan(workspace, dtype == MD_F32, B, N, Hq, d, p);
    const long units = (long)B * H * plan.cut.tiles, rows = (long)B * Hq * N;
    if (units > kMaxUnits) return fail(MD_ESHAPE, "cache4_attend: %ld tiles of query rows are too many for one call", units);
    const size_t need = attend_bytes(B, N, Hq, H, d, max_pages, page);
    const Range r[] = {{out, rows_bytes(ol, B, N, Hq, d, dtype)}, {lse, lse ? (size_t)B * Hq * N * 4 : 0}, {workspace, workspace ? need : 0},
                       {q, rows_bytes(ql, B, N, Hq, d, dtype)}, {cache, pool_bytes(p)}, {table, (size_t)B * max_pages * 4}, {len, (size_t)B * 4},
                       {q_len, q_len ? (size_t)B * 4 : 0}, {keep, keep ? (size_t)B * max_pages * page : 0}};
    rc = check_apart("cache4_attend", r, 3, 9);
    if (rc != MD_OK) return rc;
    if (!workspace || workspace_bytes < need)
        return fail(MD_EWORKSPACE, "cache4_attend: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(MD_EALIGN, "cache4_attend: workspace must be 256-byte aligned");
    const AttendArgs A{q, static_cast<const uint8_t*>(cache), table, len, q_len, keep, out, lse, p, AttendDims{B, N, G, plan.cut.tiles}, softmax_scale, ql, ol};
    // a pool beyond half of the 256 MB Infinity Cache is streamed.  us so / with plain loads: 64 x up to 4096 keys, 32 heads (680 MB) 120 / 130,
    // 16 x 4096 (300 MB) 53 / 58, 4 x 4096 (75 MB) 25.8 / 25.3
    const bool stream_once = pool_bytes(p) > (size_t)128 << 20;
    hipStream_t st = static_cast<hipStream_t>(stream);
    // A wave of a row's join adds up about eight parts, which are on their way together.  us with 4 / 8 / 16 waves: 128 parts to a unit 9.1 / 7.0 /
    // 6.6, 64 parts 7.3 / 6.3 / 6.4, 32 parts 4.7 / 5.1 / 6.4, 512 rows of 32 parts 5.4 / 6.5 / 11.6, 400 rows of 13 5.2 / 5.2 / 10.7
    const int joiners = c4_clamp((int)(kC4Blocks / units / 8), 4, 16);
#define MD_C4_ATTEND(D_, F_, NT_, S_)                                                                                                     \
    do {                                                                                                                                  \
        if (plan.cut.runs) {                                                                                                              \
            MD_LAUNCH("cache4_attend_runs", st, (cache4_attend_runs_kernel<D_, F_, NT_, S_>), kC4Blocks, 256, plan.lds, A, plan.parts);   \
            if (rows <= 2048) MD_LAUNCH("cache4_join", st, (cache4_join_kernel<D_, F_>), (int)rows, joiners * 64, 0, A, plan.parts, 16 * NT_);\
            else MD_LAUNCH("cache4_join", st, (cache4_join_tiles_kernel<D_, F_>), (int)(units * NT_), 256, 0, A, plan.parts, 16 * NT_);   \
        } else {                                                                                                                          \
            MD_LAUNCH("cache4_attend", st, (cache4_attend_kernel<D_, F_, NT_, S_>), (int)units, plan.cut.waves * 64, plan.lds, A);        \
        }                                                                                                                                 \
    } while (0)
#define MD_C4_ATTEND_S(D_, F_, NT_) do { if (stream_once) MD_C4_ATTEND(D_, F_, NT_, true); else MD_C4_ATTEND(D_, F_, NT_, false); } while (0)
#define MD_C4_ATTEND_D(D_)                                                                                                                \
    do {                                                                                                                                  \
        if (dtype == MD_F32) MD_C4_ATTEND_S(D_, true, 1);                                                                                 \
        else if (plan.cut.tile_rows == 16) MD_C4_ATTEND_S(D_, false, 1);                                                                  \
        else MD_C4_ATTEND_S(D_, false, 2);                                                                                                \
    } while (0)
    if (d == 128) MD_C4_ATTEND_D(128); else MD_C4_ATTEND_D(64);
#undef MD_C4_ATTEND_D
#undef MD_C4_ATTEND_S
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
