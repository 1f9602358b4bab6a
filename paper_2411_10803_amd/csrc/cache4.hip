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
#include "cache4_host.hpp"

namespace md {
namespace {

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
