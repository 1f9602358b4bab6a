/*
 * mustdrop.h -- C ABI of the MustDrop token-reduction library for AMD MI355X (gfx950).
 *
 * Three entry points, one per stage of the method (Liu et al., "Multi-Stage
 * Vision Token Dropping", CVPR 2025):
 *   mustdrop_encode_merge    Sec. 3.3  Local Spatial Merging (Eq. 5) + Key Retaining (Eq. 6-7)
 *   mustdrop_prefill_filter  Sec. 3.4  dual-attention filtering (Eq. 8-10) + token drop
 *   mustdrop_decode_evict    Sec. 3.5  output-aware cache policy, one decode step
 * and, behind them, a paged cache held in 4 bits with the attention that reads it, all of it or the pages that a cheap score
 * chooses (mustdrop_cache4_*), and the rotation of queries and keys by positions with several axes (mustdrop_rotate).
 *
 * Conventions common to all calls
 *   - Every data pointer is DEVICE memory owned by the caller (inputs, outputs and the workspace).
 *     The entry points of this header allocate nothing, free nothing and keep no state between
 *     calls, with these exceptions, all stated here: the thread-local text behind
 *     mustdrop_last_error(); the static device buffer of mustdrop_encode_merge_noalloc and the
 *     address of it that the library looks up once per device (see there); and, while a caller
 *     has switched on the benchmarking aid declared in mustdrop_bench.h (a separate header, not
 *     needed to use the method), one pair of HIP events per kernel launch.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL = the null stream).  No
 *     call synchronises with the host; variable-length results are reported through device-side
 *     count arrays and the outputs are padded to a static capacity.
 *   - Tensors are row-major with the last dimension contiguous.  Base pointers of the large
 *     tensors must be 16-byte aligned and their rows (D, dc, d, C elements) a multiple of 16 bytes.
 *   - Indices are int32, 0-based, in the coordinates of that call's input; index lists ascend.
 *   - Inputs are never written, except what is marked in/out and the in/out state of mustdrop_decode_evict.
 *   - Return value: MD_OK or an error code.  Argument errors are detected on the host before any
 *     kernel is launched; mustdrop_last_error() returns a thread-local description.
 *   - `workspace` must hold at least mustdrop_<stage>_workspace_bytes(...) bytes, 256-byte aligned.
 *     Calls that share a workspace must be ordered on one stream.  Calls that share neither a
 *     workspace nor an output or state buffer may overlap in time (several streams): a caller with
 *     independent batches can keep two of them in flight.
 */
#ifndef MUSTDROP_H
#define MUSTDROP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types and modes cross the boundary as plain ints (a caller may hand over any value: one
 * that names nothing is an error code, never undefined behaviour). */
typedef int md_dtype;
enum { MD_F32 = 0, MD_BF16 = 1 };

typedef enum {
    MD_OK = 0,
    MD_EINVAL = 1,      /* null required pointer, non-positive size, value out of range */
    MD_ESHAPE = 2,      /* shapes that do not fit together or that no kernel supports   */
    MD_EALIGN = 3,      /* pointer or row size not 16-byte aligned                      */
    MD_EALIAS = 4,      /* an output overlaps an input                                  */
    MD_EWORKSPACE = 5,  /* workspace missing or too small                               */
    MD_EDTYPE = 6,      /* unknown dtype / mode enum                                    */
    MD_EHIP = 7         /* the HIP runtime reported an error at launch                  */
} md_status;

typedef int md_filter_mode;
enum { MD_FILTER_BUDGET = 0, MD_FILTER_THRESHOLD = 1 };

/* Thread-local text of the last error returned on this thread ("" if none). */
const char* mustdrop_last_error(void);

/* Library version, major*100 + minor (2: mustdrop_prefill_filter takes row_lse; 3: the cache held in 4 bits). */
int mustdrop_version(void);

/* ------------------------------------------------------------------------------------------
 * Stage 1 -- vision encoding (Sec. 3.3).
 *
 * Key Retaining (Eq. 6-7): a_cls[j] = mean over the Hc heads of softmax_j(q_cls . k_j / sqrt(dc)),
 * the softmax running over all 1+M keys (key 0 is the [CLS] key, whose own probability is
 * discarded).  The key set O is the `key_budget` valid tokens with the largest a_cls (ties: lower
 * index).  Local Spatial Merging (Eq. 5): the T x Hg x Wg grid is cut into non-overlapping
 * kt x kh x kw windows (where the window does not divide the grid, the windows at the far border are
 * clipped to the grid and hold fewer tokens); S = mean over unordered member pairs of their cosine
 * similarity (zero-norm member: cosine 0).  A window merges iff S > tau, it has at least two valid members and none of
 * them is in O; its members are replaced by one token: the mass-weighted mean of the members, with
 * mass = sum of member masses, at the position of the lowest member index.  Survivors are written
 * in ascending original index.
 *
 *   x          [B, M, D]          M = T*Hg*Wg, token index = (t*Hg + y)*Wg + x; dtype x_dtype
 *   q_cls      [B, Hc, dc]        CLS query;   k_cls [B, 1+M, Hc, dc] keys (row 0 = CLS key);
 *                                 dtype qk_dtype; both NULL iff key_budget == 0; dc a power of two
 *   mass_in    [B, M] f32 or NULL (all ones)      valid [B, M] u8 or NULL (all valid)
 *   tau        threshold on the MEAN pairwise cosine (the paper's ordered-pair sum is
 *              ws*(ws-1) times the mean, ws = kt*kh*kw)
 *   out_x      [B, M, D]  dtype x_dtype; rows >= out_count[b] are left untouched.  Unmerged rows
 *              are bit-identical copies; merged rows are accumulated in fp32 and rounded to nearest even
 *   out_index, out_mass, out_is_key [B, M]; out_valid [B, M] u8 (1 for slots < out_count[b]; may be NULL)
 *   out_count  [B]
 *   key_index  [B, key_budget] ascending, padded with -1 if fewer valid tokens exist
 *   a_cls_out  [B, M] f32 or NULL;  window_sim_out [B, W] f32 or NULL,
 *              W = ceil(T/kt)*ceil(Hg/kh)*ceil(Wg/kw), window index = (wt*ceil(Hg/kh) + wy)*ceil(Wg/kw) + wx
 *
 * Limits: kt*kh*kw <= 16; D*elt and dc*elt multiples of 16 bytes.
 * Errors: MD_EINVAL, MD_ESHAPE (window too large, Hc*dc unusable), MD_EALIGN, MD_EALIAS (out_x overlaps x), MD_EWORKSPACE, MD_EDTYPE, MD_EHIP.
 */
size_t mustdrop_encode_merge_workspace_bytes(int B, int T, int Hg, int Wg, int Hc, int kt, int kh, int kw);

int mustdrop_encode_merge(
    const void* x, md_dtype x_dtype,
    const void* q_cls, const void* k_cls, md_dtype qk_dtype,
    const float* mass_in, const uint8_t* valid,
    int B, int T, int Hg, int Wg, int D, int Hc, int dc,
    int kt, int kh, int kw, float tau, int key_budget,
    void* out_x, int32_t* out_index, float* out_mass, uint8_t* out_is_key, uint8_t* out_valid,
    int32_t* out_count, int32_t* key_index,
    float* a_cls_out, float* window_sim_out,
    void* workspace, size_t workspace_bytes, void* stream);

/* mustdrop_encode_merge for callers that cannot allocate device memory or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, outputs and
 * errors as mustdrop_encode_merge, minus `workspace` / `workspace_bytes`: the scratch memory is a static
 * device array of MUSTDROP_STATIC_SCRATCH_BYTES inside the library (each GPU the library runs on holds
 * one until the process ends).  The call allocates and frees nothing.  A shape whose
 * mustdrop_encode_merge_workspace_bytes(...) exceeds the static buffer is rejected with MD_EWORKSPACE
 * (8 MiB covers up to 16 samples of 2880 tokens, or 4 of 4608, with 16 CLS heads).  The first call on
 * a device looks up the array's device address; do that call outside a graph capture.  All calls on one
 * GPU share the array, which keeps the previous call's contents (nothing in it needs clearing): calls
 * that overlap in time on one GPU race -- order them on one stream. */
#define MUSTDROP_STATIC_SCRATCH_BYTES (8u << 20)

int mustdrop_encode_merge_noalloc(
    const void* x, md_dtype x_dtype,
    const void* q_cls, const void* k_cls, md_dtype qk_dtype,
    const float* mass_in, const uint8_t* valid,
    int B, int T, int Hg, int Wg, int D, int Hc, int dc,
    int kt, int kh, int kw, float tau, int key_budget,
    void* out_x, int32_t* out_index, float* out_mass, uint8_t* out_is_key, uint8_t* out_valid,
    int32_t* out_count, int32_t* key_index,
    float* a_cls_out, float* window_sim_out, void* stream);

/* Stage 1 with the key set in the printed form of Eq. 7: O = { j : a_cls[j] > mu }.  The paper only says
 * that mu is adaptive and depends on a_cls; this library reads it as mu = mean + key_lambda * std of
 * a_cls over the valid tokens (population standard deviation, fp32).  Everything else is
 * mustdrop_encode_merge.  key_cap >= 0 is the capacity of key_index per sample ([B, key_cap], may be
 * NULL if 0): the first key_cap members of O in ascending order, the rest -1; key_count [B] (required)
 * receives |O|, which may exceed key_cap.  q_cls and k_cls are always required. */
int mustdrop_encode_merge_adaptive(
    const void* x, md_dtype x_dtype,
    const void* q_cls, const void* k_cls, md_dtype qk_dtype,
    const float* mass_in, const uint8_t* valid,
    int B, int T, int Hg, int Wg, int D, int Hc, int dc,
    int kt, int kh, int kw, float tau, float key_lambda, int key_cap,
    void* out_x, int32_t* out_index, float* out_mass, uint8_t* out_is_key, uint8_t* out_valid,
    int32_t* out_count, int32_t* key_index, int32_t* key_count,
    float* a_cls_out, float* window_sim_out,
    void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Stage 2 -- prefill, one LLM layer (Sec. 3.4).  Sequence per sample: [vision 0..Mv-1 | text 0..N-1]
 * (Sec. 3.1, prefilling: X = {V_1..V_M, T_1..T_N}), L = Mv + N.
 *
 * a[i][j] = mean over heads of the softmax probability of text row i on vision column j; each
 * text row's softmax runs over the valid vision keys and the text keys 0..i (causal).
 * V_j = sum_i a[i][j] (Eq. 8), I_j = max_i a[i][j] (Eq. 10), G = sum_j V_j (Eq. 9, valid j only).
 *   MD_FILTER_THRESHOLD: drop j iff V_j <= gamma*G and I_j < alpha and j is not a key token.
 *   MD_FILTER_BUDGET:    keep the key tokens, then the (budget - #keys) other valid tokens with
 *                        the largest s_j = max(V_j/(gamma*G), I_j/alpha) (ties: lower index);
 *                        gamma, alpha > 0 required.
 * Token drop: rows [kept vision tokens ascending | text rows 0..txt_len-1] of hidden, k and v are
 * copied bit for bit to the outputs.
 *
 *   q_txt      [B, N, H, d] bf16   queries of the text tokens
 *   k, v       [B, L, H, d] bf16;  hidden [B, L, C] bf16
 *   vis_valid  [B, Mv] u8 or NULL; txt_len [B] i32 or NULL (= N; text is padded at the tail);
 *   is_key     [B, Mv] u8 or NULL (no key tokens)
 *   row_lse    [B, H, N] f32 or NULL.  The scores a[i][j] are a by-product of the layer's own attention
 *              (Sec. 3.4); a flash-style attention kernel keeps, per head and query row, the natural-log
 *              sum of exp(softmax_scale * q.k) over the keys that row sees.  Given those values for the text rows
 *              (over the valid vision keys and the text keys 0..i, with this call's softmax_scale), the
 *              library skips its own pass over K for the softmax normalisers and reads K once instead
 *              of twice.  Entries of rows >= txt_len are ignored.  NULL: the library computes them.
 *   Rcap       capacity, in rows, of the kept-vision part of the outputs (>= budget in budget mode;
 *              use Mv in threshold mode).  The caller must size it for max(budget, #keys).
 *   hidden_out [B, Rcap+N, C], k_out, v_out [B, Rcap+N, H, d]; rows >= out_len[b] untouched
 *   kept_index [B, Rcap] (entries >= min(kept_count, Rcap) untouched)
 *   kept_count [B]   number of vision tokens the rule keeps; if it exceeds Rcap only the first
 *                    Rcap (lowest indices) are stored -- an overflow the caller can detect
 *   out_len    [B] or NULL   = min(kept_count, Rcap) + txt_len: live rows of the outputs
 *   out_ids    [B, Rcap+N] i32 or NULL: original sequence position of every output row (vision index j,
 *              or Mv+i for text row i; -1 for rows that are not live) -- usable as the decode stage's ids
 *   out_protect[B, Rcap+N] u8 or NULL: 1 for key tokens and text rows (the decode stage's protect flags)
 *   score_global, score_indiv [B, Mv] f32 or NULL: V_j and I_j (0 for invalid tokens)
 *
 * Limits: d in {64, 128}; N <= 1024 (tuned for N <= 128: a longer prompt is cut into groups of up to 128
 * text rows, and every group goes over K in both sweeps); H <= 128; softmax_scale positive
 * and finite; C*2 and H*d*2 multiples of 16 bytes.
 */
size_t mustdrop_prefill_filter_workspace_bytes(int B, int Mv, int N, int H, int Rcap);

int mustdrop_prefill_filter(
    const void* q_txt, const void* k, const void* v, const void* hidden,
    const uint8_t* vis_valid, const int32_t* txt_len, const uint8_t* is_key, const float* row_lse,
    int B, int Mv, int N, int H, int d, int C,
    float softmax_scale, md_filter_mode mode, int budget, float gamma, float alpha,
    int Rcap,
    void* hidden_out, void* k_out, void* v_out,
    int32_t* kept_index, int32_t* kept_count, int32_t* out_len, uint8_t* out_protect, int32_t* out_ids,
    float* score_global, float* score_indiv,
    void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Stage 3 -- decode, one step of one layer (Sec. 3.5; decode attention as in Eq. 4).
 *
 * a_t[j] = mean over heads of softmax_j(softmax_scale * q_h . k_jh) over the live entries
 * j < len[b]; acc[j] <- decay*acc[j] + a_t[j].  If len[b] > budget, the protected entries and the
 * (budget - #protected) unprotected entries with the largest acc stay (ties: lower id); the rest
 * are evicted.  With protect = the set S_few and budget = |S_few| this is the paper's static
 * policy.  The cache is compacted by hole filling: survivors sitting at slots >= new_len move, in
 * ascending slot order, into the evicted slots < new_len, in ascending slot order; K/V rows move
 * bit for bit together with their acc / ids / protect entries.
 *
 *   q        [B, H, d] bf16             query of the token being generated
 *   k_cache, v_cache [B, Lcap, H, d] bf16   in/out
 *   acc      [B, Lcap] f32 (>= 0: entries are ranked by the bit pattern of their score), ids [B, Lcap] i32
 *            (in [0, 2^31 - 2], unique per sample), protect [B, Lcap] u8, len [B] i32: in/out
 *   decay    >= 0 (MD_EINVAL otherwise), so that the running scores stay non-negative
 *   evicted_ids [B, Lcap] or NULL: ids of the evicted entries in ascending (pre-compaction) slot order
 *   evicted_count [B] or NULL
 *
 * Limits: d a power of two in [8, 512]; H <= 1024 (with d = 64 or 128 and rows of at most 16 KiB the scores
 * come from the streaming kernel; the selection then runs in registers where Lcap <= 8192 and H is 4, 8, 16
 * or 32, or another multiple of four with 4*Lcap + 512*H <= 65536; other shapes take the general kernels).
 * MD_EALIAS: q, the two caches, acc, ids, protect, len, the optional outputs and the workspace must be
 * pairwise disjoint.
 */
size_t mustdrop_decode_evict_workspace_bytes(int B, int Lcap, int H);

int mustdrop_decode_evict(
    const void* q, void* k_cache, void* v_cache,
    float* acc, int32_t* ids, uint8_t* protect, int32_t* len,
    int B, int Lcap, int H, int d,
    float softmax_scale, float decay, int budget,
    int32_t* evicted_ids, int32_t* evicted_count,
    void* workspace, size_t workspace_bytes, void* stream);

/* Appends one entry per sample at slot len[b] (Eq. 3: K <- Concat(K, x_i W_k), same for V):
 * copies k_new[b], v_new[b] ([B, H, d] bf16), sets acc = 0, ids = new_id, protect = protect_new,
 * len[b] += 1.  Samples whose cache is full (len[b] == Lcap) are left unchanged.  Device-side,
 * asynchronous, so a decode loop needs no host round trip. */
int mustdrop_decode_append(
    const void* k_new, const void* v_new,
    void* k_cache, void* v_cache,
    float* acc, int32_t* ids, uint8_t* protect, int32_t* len,
    int B, int Lcap, int H, int d, int32_t new_id, int protect_new, void* stream);

/* ------------------------------------------------------------------------------------------
 * Stage 3, the static policy as printed (Sec. 3.5): from the shallow layers on, the caches store only
 * the vision tokens of the set S_few (besides the text and what was generated) -- nothing is scored.
 * keep[b][j] != 0 marks the entries j < len[b] that stay.  The caches of all n_layers layers are
 * compacted in one call by the hole filling of mustdrop_decode_evict (the kept entries at slots
 * >= new_len move, in ascending order, into the dropped slots < new_len, in ascending order), so every
 * layer holds the same entry in the same slot and ids / protect / acc describe all of them.
 *
 *   k_cache, v_cache [n_layers, B, Lcap, H, d] bf16, in/out (device)
 *   keep     [B, Lcap] u8, read only (entries >= len[b] are ignored)
 *   acc      [B, Lcap] f32 in/out, or NULL;  ids [B, Lcap] i32, protect [B, Lcap] u8, len [B] i32: in/out
 *   evicted_ids [B, Lcap] or NULL: ids of the dropped entries in ascending slot order;
 *   evicted_count [B] or NULL
 *   workspace: mustdrop_decode_evict_workspace_bytes(B, Lcap, H) bytes, 256-byte aligned
 * Limits and errors as for mustdrop_decode_evict; n_layers in [1, 65535].
 */
int mustdrop_decode_keep(
    void* k_cache, void* v_cache, const uint8_t* keep,
    float* acc, int32_t* ids, uint8_t* protect, int32_t* len,
    int n_layers, int B, int Lcap, int H, int d,
    int32_t* evicted_ids, int32_t* evicted_count,
    void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Other memory layouts of Q, K and V (the tensors of Eq. 3-4; what the stages compute is unchanged).
 *
 * The entry points above take the token-major layout [B, tokens, H, d].  The *_strided twins below
 * take, per tensor group, the ELEMENT strides of the batch, token and head axes; the d elements of
 * one (sample, token, head) stay contiguous.  A head-major cache [B, H, tokens, d] is
 * {H*tokens*d, d, tokens*d}; a token-major one with padded rows {tokens*pitch, pitch, d}.
 * A NULL layout means dense token-major, and a call whose layouts are all dense token-major takes
 * exactly the path of the plain entry point.  For other layouts the score kernels run with strided
 * addressing and the row copies gather a token's row head slice by head slice (d*2 contiguous
 * bytes at a time).
 *
 * Every stride must be a positive multiple of 8 elements (16 bytes), and the three axes must nest
 * without overlap: sorted by stride, stride[0] >= d, stride[1] >= stride[0]*extent[0],
 * stride[2] >= stride[1]*extent[1] (else MD_ESHAPE).  The caller's allocation must cover
 * (B-1)*batch + (tokens-1)*token + (H-1)*head + d elements from the base pointer.
 * All other arguments, outputs, limits and errors are those of the plain entry point.
 */
typedef struct {
    int64_t batch;   /* elements between consecutive samples       */
    int64_t token;   /* elements between consecutive tokens/slots  */
    int64_t head;    /* elements between consecutive heads         */
} md_kv_layout;      /* host memory; read during the call only     */

/* q_layout: q_txt over N tokens; kv_layout: k and v over L = Mv+N tokens (one layout for both);
 * kv_out_layout: k_out and v_out over Rcap+N rows.  hidden and hidden_out stay [B, rows, C]. */
int mustdrop_prefill_filter_strided(
    const void* q_txt, const void* k, const void* v, const void* hidden,
    const uint8_t* vis_valid, const int32_t* txt_len, const uint8_t* is_key, const float* row_lse,
    int B, int Mv, int N, int H, int d, int C,
    float softmax_scale, md_filter_mode mode, int budget, float gamma, float alpha,
    int Rcap,
    void* hidden_out, void* k_out, void* v_out,
    int32_t* kept_index, int32_t* kept_count, int32_t* out_len, uint8_t* out_protect, int32_t* out_ids,
    float* score_global, float* score_indiv,
    const md_kv_layout* q_layout, const md_kv_layout* kv_layout, const md_kv_layout* kv_out_layout,
    void* workspace, size_t workspace_bytes, void* stream);

/* cache_layout: k_cache and v_cache over Lcap slots.  q, k_new, v_new stay [B, H, d]. */
int mustdrop_decode_evict_strided(
    const void* q, void* k_cache, void* v_cache,
    float* acc, int32_t* ids, uint8_t* protect, int32_t* len,
    int B, int Lcap, int H, int d,
    float softmax_scale, float decay, int budget,
    int32_t* evicted_ids, int32_t* evicted_count,
    const md_kv_layout* cache_layout,
    void* workspace, size_t workspace_bytes, void* stream);

int mustdrop_decode_append_strided(
    const void* k_new, const void* v_new,
    void* k_cache, void* v_cache,
    float* acc, int32_t* ids, uint8_t* protect, int32_t* len,
    int B, int Lcap, int H, int d, int32_t new_id, int protect_new,
    const md_kv_layout* cache_layout, void* stream);

/* layer_stride: elements between the caches of consecutive layers (ignored when n_layers == 1;
 * a positive multiple of 8 that is at least the extent of one layer's cache, else MD_ESHAPE). */
int mustdrop_decode_keep_strided(
    void* k_cache, void* v_cache, const uint8_t* keep,
    float* acc, int32_t* ids, uint8_t* protect, int32_t* len,
    int n_layers, int B, int Lcap, int H, int d,
    int32_t* evicted_ids, int32_t* evicted_count,
    const md_kv_layout* cache_layout, int64_t layer_stride,
    void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * A cache held in 4 bits, in pages (the cache of Eq. 3-4 in a smaller form).  What the stages above keep -- the rows of
 * mustdrop_prefill_filter (k_out, v_out, with out_len rows per sample), then one entry per step -- goes into pages of a pool
 * that all samples share, and attention reads the pages.
 *
 * Numbers.  32 consecutive channels of one token and head are 32 four-bit numbers (bit 3: sign, bits 0-2: index of the magnitude
 * among 0, 0.5, 1, 1.5, 2, 3, 4, 6) times one scale 2^e.  With a the largest magnitude of the 32 and k = floor(log2 a): e = k - 2,
 * or k - 1 where a >= 1.75 * 2^k (a is then rounded to 6 at most and not cut down to it), at least -100 and at most 125, and -100
 * where a = 0.  x becomes the nearest value to x / 2^e, of two as near the one of the even index, and 6 where it is more.  The scale
 * is the byte e + 127; a group with an infinity or a NaN has 255 and all of it reads as NaN.  With 3.5 * 2^-100 <= a < 7 * 2^125
 * (2.8e-30 to 2.9e38) a value is off by at most a fifth of a, and by at most a fifth of itself where it is no smaller than a / 4.
 * Below, where e stays at -100, values are off by up to 2^-101, and those up to 2^-102 read as 0; above, where e stays at 125, what
 * is beyond 6 * 2^125 reads as that (off by up to a quarter of itself), and the others are off by a fifth of a at most.
 *
 * Pool.  [n_pages, H] pieces of page * (d + d/16) bytes (mustdrop_cache4_bytes in all), each one after the other
 *   K codes [page, d/2] (channel 2i in the low half of byte i), K scales [page, d/32],
 *   V codes [page/4, 16, 4, d/32] (four tokens side by side: their bytes of the d/16 channels of each sixteenth of the row),
 *   V scales [page/4, d/32, 4].
 * Nothing in the pool needs clearing: what lies behind a sample's length is not used, whatever it holds.
 *
 * Block table.  table [B, max_pages] i32: entry e of sample b names the page of its entries e*page .. e*page + page-1.  Entries
 * from ceil(len/page) on may hold anything and change no result; calls may read them, and in the pages that they name, so all
 * of the table has to be memory that can be read.  slot = page number * page + place in the page, i32; -1: none.  A page number
 * outside the pool names no page: its entries take no part in attention, its rows are not read out; a slot outside the pool is
 * not written.
 *
 * The stages above do not read this cache.  mustdrop_decode_evict and mustdrop_decode_keep take dense rows: read the cache out, evict,
 * write what is left.  The `keep` of the attention comes from the caller; nothing here makes one from the pages.
 *
 * Limits of the cache4 calls: d in {64, 128}; page a power of two from 16 to 256; n_pages * page < 2^31,
 * max_pages * page < 2^30; a pool of at most 256 GiB; H <= 65535; rows in MD_BF16 or MD_F32, fewer than 2^28 - 15 of them
 * (B*N) in or out in a call; base pointers 16-byte aligned.  md_kv_layout as above
 * (elements of the rows' type); NULL = dense token-major.  MD_EALIAS goes by a tensor's first and last element: an output whose rows
 * lie between those of another tensor (K and V side by side in one buffer) is refused, inputs may lie so, and so may the q_out of
 * mustdrop_cache4_append between other rows (see mustdrop_rotate).
 */
size_t mustdrop_cache4_bytes(int n_pages, int page, int H, int d);      /* 0 for sizes that no call takes */

/* Block tables and slots from lengths: every sample b is to hold new_len[b] entries, where it held len[b].  Both are taken as 0
 * where negative and as max_pages*page where larger.  A sample holds ceil(length / page) pages.  Pages that are not needed any
 * more go onto the stack of free pages, in the order of samples and entries, the first one uppermost; then the pages that are
 * needed come off its top, in the order of samples and entries.  A call that takes back what another one did therefore leaves
 * the stack as it was.
 *   new_len  [B];  len [B] in/out;  table [B, max_pages] in/out (entries that are not taken in this call stay as they are,
 *            released ones among them)
 *   free_pages [n_pages] in/out: the stack, its bottom first;  n_free [1] in/out: its height
 *   slots    [B, N]: slots of the new entries, slots[b][i] that of entry len[b] + i (len as it was), -1 from new_len[b] on; NULL if N = 0
 *   missing  [1]: pages that the pool is short of.  If not 0, nothing else is changed, and the slots are all -1.
 * One page per entry of the stack and the tables: a page named twice is handed out twice.  Errors: MD_EINVAL, MD_ESHAPE
 * (limits, B > 65535, N > 2^30, B * max_pages + n_pages > 2^31 - 8193), MD_EALIAS, MD_EALIGN, MD_EWORKSPACE, MD_EHIP. */
size_t mustdrop_cache4_pages_workspace_bytes(int B);

int mustdrop_cache4_pages(
    const int32_t* new_len, int32_t* len, int32_t* table, int32_t* free_pages, int32_t* n_free, int32_t* slots, int32_t* missing,
    int B, int max_pages, int n_pages, int page, int N, void* workspace, size_t workspace_bytes, void* stream);

/* Rows into the cache: k_new, v_new [B, N, H, d] (dtype; rows_layout), row (b, i) to slots[b][i], rows without a slot not at all.
 * No two rows of a call may have the same slot (the slot then holds parts of both).  Errors: MD_EINVAL, MD_ESHAPE, MD_EDTYPE,
 * MD_EALIGN, MD_EALIAS (the rows or slots overlap the cache), MD_EHIP. */
int mustdrop_cache4_write(
    const void* k_new, const void* v_new, md_dtype dtype, const int32_t* slots, void* cache,
    int B, int N, int H, int d, int n_pages, int page, const md_kv_layout* rows_layout, void* stream);

/* Rows out of the cache, as the dense stages take them (mustdrop_decode_evict): k_out, v_out [B, N, H, d] (dtype; rows_layout),
 * row (b, i) the entry first[b] + i; rows of entries outside 0 .. len[b]-1 are left untouched.  first [B] i32 or NULL (0).  The values
 * are exact in bf16, but for magnitudes beyond its range (none that the write makes).  Errors as for mustdrop_cache4_write. */
int mustdrop_cache4_read(
    const void* cache, const int32_t* table, const int32_t* len, const int32_t* first, void* k_out, void* v_out, md_dtype dtype,
    int B, int N, int H, int d, int n_pages, int page, int max_pages, const md_kv_layout* rows_layout, void* stream);

/* Attention over the cache (Eq. 4), for the last q_len[b] entries of every sample: query row i stands at entry
 * len[b] - q_len[b] + i and sees the entries up to its own, but for those that `keep` leaves out.  N = 1 is the decode step, a few
 * rows a draft, many a piece of a prompt (whose entries are written before the call).  Query head h reads K/V head h / (Hq/H).
 *   out = sum_j p_j v_j,  p = softmax_j(softmax_scale * q . k_j);  lse = the natural logarithm of the sum of exp(softmax_scale * q . k_j)
 *   q        [B, N, Hq, d] (dtype; q_layout);  Hq a multiple of H
 *   q_len    [B] i32 or NULL (= N); taken as 0 where negative, as N where larger;  len [B] i32, likewise within 0 .. max_pages*page
 *   keep     [B, max_pages*page] u8 or NULL (all): entries with keep 0 are seen by no row (they may hold anything)
 *   out      [B, N, Hq, d] (dtype; out_layout), rows >= q_len[b] untouched;  lse [B, Hq, N] f32 or NULL, likewise
 * softmax_scale is positive and finite, times log2(e) too.  A row that sees no entry gets out = 0 and lse = -infinity, as does one
 * with all scores below -2e38.  A row whose query or scores are no numbers, or with a score beyond 2.3e38, is NaN, and so are the
 * channels of a group of V that is, in the rows that see it; no other row is.  Scores, sums and the running maximum are fp32 (the sum of
 * p_j v_j is up to 2^12 times as large before it is divided: a V below 8e34 / len cannot overflow); a probability enters the product
 * with V as a sum of bf16 parts that carries 24 bits for MD_F32 and 16 for MD_BF16.  An fp32 query is a sum of three bf16 parts: all of its
 * 24 bits from 2^-110 on, what is above 2^-134 below that; beyond 3.39e38 its row is NaN.  Two calls on the same inputs with tables of
 * the same width give the same bits.  The (N * Hq/H) rows of a sample and K/V head are taken 16 at a time, or 32 for MD_BF16 where
 * they are more than 16 and there are more than 512 tiles of 16 in the call; a call takes fewer than 2^23 such tiles.  Errors: MD_EINVAL,
 * MD_ESHAPE, MD_EDTYPE, MD_EALIGN (keep 4-byte aligned), MD_EALIAS, MD_EWORKSPACE, MD_EHIP. */
size_t mustdrop_cache4_attend_workspace_bytes(int B, int N, int Hq, int H, int d, int max_pages, int page);

int mustdrop_cache4_attend(
    const void* q, md_dtype dtype, const void* cache, const int32_t* table, const int32_t* len, const int32_t* q_len, const uint8_t* keep,
    int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, float softmax_scale,
    void* out, float* lse, const md_kv_layout* q_layout, const md_kv_layout* out_layout,
    void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Rotation of queries and keys by their positions.  A token of an image or a video has a place on several axes (time, height, width),
 * and what the stages above keep are rows whose places are not consecutive any more.
 *
 * Of a row's d channels the first 2 * pairs turn in pairs: pair i is channels (i, i + pairs), or (2i, 2i + 1) where `adjacent`; the
 * others stay.  Pair i has an axis; with p the row's position on it and (c, s) = table[p][i], (x, y) becomes (x c - y s, y c + x s), or
 * with -s in the place of s where `inverse` (the gradient; where c^2 + s^2 = 1 the way back, too).  In fp32: the products are rounded, then
 * their sum, then the result to the rows' type.  What the angles are (base, scaling, any factor) is the table's business.
 *   pairs      a multiple of 4 (8 for mustdrop_cache4_append), 2 * pairs <= d
 *   axes       1 to 4;  axis[i] < axes for i < pairs
 *   table      [n_pos, pairs, 2] f32: cosine and sine of each position's angles
 *   positions  [axes, B, L] i32;  index [B, N] i32 or NULL: row (b, i) is at positions[.][b][index[b][i]], or [i] without index (then
 *              L >= N).  A position outside 0 .. n_pos-1 turns its pairs into NaN, an index outside 0 .. L-1 all pairs of its row.
 */
typedef struct md_rotary {
    int32_t pairs, axes, adjacent;
    uint8_t axis[128];
} md_rotary;

/* Rows turned: q [B, N, Hq, d] into q_out, and k [B, N, H, d] into k_out in the same launch (k = k_out = NULL: only q).  An output may be
 * its input, with the same layout; no other overlap.  Rows may lie between other rows: q and k as views of one projection's output, turned in
 * place, share no byte (MD_EALIAS goes by bytes where the strides of batch, tokens and heads are the same, else by first and last
 * element).  rows [B] i32 or NULL (= N): rows (b, i) with i >= rows[b] are not read and
 * not written.  d a multiple of 8, at most 256; layouts as md_kv_layout, NULL = dense token-major; B * N <= 2^28 - 16, and at most
 * 2^31 - 512 pieces of 16 channels (of 8 with MD_F32, or where d or 2 * pairs is no multiple of 16) in all heads of all rows.  Errors:
 * MD_EINVAL, MD_ESHAPE, MD_EDTYPE, MD_EALIGN, MD_EALIAS, MD_EHIP. */
int mustdrop_rotate(
    const void* q, const void* k, md_dtype dtype, const int32_t* positions, const int32_t* index, const float* table, const int32_t* rows,
    int B, int N, int L, int Hq, int H, int d, int n_pos, const md_rotary* rotary, int inverse,
    void* q_out, void* k_out,
    const md_kv_layout* q_layout, const md_kv_layout* k_layout, const md_kv_layout* q_out_layout, const md_kv_layout* k_out_layout,
    void* stream);

/* Rows into the cache held in 4 bits (mustdrop_cache4_write), k_new [B, N, H, d] turned on the way: the turned fp32 numbers are what is
 * rounded to 4 bits.  q [B, N, Hq, d] is turned too, into q_out (which may be q, with the same layout), in the same launch; q = q_out =
 * NULL: no queries.  A row whose slot names no place of the pool takes no part, its query neither.  k_new and v_new have rows_layout;
 * no two rows of a call may have the same slot.  Errors as for mustdrop_cache4_write and mustdrop_rotate. */
int mustdrop_cache4_append(
    const void* q, const void* k_new, const void* v_new, md_dtype dtype, const int32_t* positions, const int32_t* index, const float* table,
    const int32_t* slots, void* cache,
    int B, int N, int L, int Hq, int H, int d, int n_pos, int n_pages, int page, const md_rotary* rotary,
    void* q_out, const md_kv_layout* q_layout, const md_kv_layout* rows_layout, const md_kv_layout* q_out_layout, void* stream);

/* ------------------------------------------------------------------------------------------
 * Attention over a part of the cache held in 4 bits: over the pages that a cheap score chooses for each token and K/V head.  For pools,
 * block tables and their limits see above.
 *
 * Bounds of a page's keys, per head.  With a the largest magnitude among the page's keys and e = floor(log2 a) - 6 (a = 0: -126), at
 * least -126: bounds [n_pages, H, 2, d] i8, every channel's largest value over 2^e rounded up, then every channel's smallest one rounded
 * down (within -96 and 96); scales [n_pages, H] u8 the byte e + 127, or 255 where a group of the page's keys has a scale beyond 252 (the
 * write makes no other than 255: a key that is no number), whose bounds are then 0.  Values of groups whose scale is at least an eighth of
 * the largest one's are held exactly.
 */

/* Bounds of the pages that hold the entries first[b] .. min(first[b] + N, len[b]) - 1 of every sample, each over all of the page's
 * entries below len[b]: what else the page holds does not count.  A page that several entries of the tables name has to be as full
 * for each of them (its bounds may be parts of theirs otherwise).  first [B] i32 or NULL (0); negative ones are taken as 0.
 * Errors: MD_EINVAL, MD_ESHAPE (limits, more than 2^25 pages and heads to go through), MD_EALIGN, MD_EALIAS, MD_EHIP. */
int mustdrop_cache4_bounds(
    const void* cache, const int32_t* table, const int32_t* len, const int32_t* first, int8_t* bounds, uint8_t* scales,
    int B, int N, int H, int d, int n_pages, int page, int max_pages, void* stream);

/* The pages that a token's attention is to read, for each of the last q_len[b] entries of every sample (which see entries as in
 * mustdrop_cache4_attend) and each K/V head.
 * The G = Hq / H queries of a token and K/V head become whole numbers: with a their largest magnitude, those of 2^(floor(log2 a) - 6),
 * the nearest (of two as near the even one), within -127 and 127; all 0 where a is 0 or no finite number.  A page's score is
 *   2^e * sum over the G queries and the channels of max(q * largest, q * smallest)
 * with the page's bounds, summed in whole numbers and rounded to fp32 once: no key of the page has a larger sum of its scores with the
 * rounded queries.  The choice does not know the `keep` of the attention: a page keeps its score and its place in the budget whatever a mask leaves
 * out of it, all of its entries too (a copy of the block table that names no page there keeps such pages out of the choice).  Where scales is 255 the score is +infinity; where the table names no page, -infinity.
 * Of the P pages that the token sees, the first first_pages and the last last_pages are taken, then those with the highest scores, of
 * equal ones the first, until there are min(budget, P).
 *   q [B, N, Hq, d] (dtype; q_layout);  q_len [B] i32 or NULL (= N)
 *   chosen [B, N, H, budget] i32: entries of the block table in ascending order, then -1; rows i >= q_len[b] untouched
 * first_pages, last_pages >= 0 with a sum of at most budget; budget <= 2^26; max_pages <= 2^23 - 128; G <= 1024 (sums have 31 bits),
 * N * G <= 2^20.  The same inputs give the same pages, whatever else differs.
 * Errors: MD_EINVAL, MD_ESHAPE (limits, more than 2^23 - 1 tokens and heads), MD_EDTYPE, MD_EALIGN, MD_EALIAS, MD_EWORKSPACE, MD_EHIP. */
size_t mustdrop_cache4_choose_workspace_bytes(int B, int N, int Hq, int H, int d, int max_pages, int page);

int mustdrop_cache4_choose(
    const void* q, md_dtype dtype, const int8_t* bounds, const uint8_t* scales, const int32_t* table, const int32_t* len, const int32_t* q_len,
    int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, int first_pages, int last_pages, int budget,
    int32_t* chosen, const md_kv_layout* q_layout, void* workspace, size_t workspace_bytes, void* stream);

/* mustdrop_cache4_attend over chosen pages: query row (b, i) sees, for K/V head h, those of the entries that it sees there which lie in
 * the pages that chosen[b][i][h][0 .. budget-1] names.  An entry of chosen that is not in 0 .. max_pages-1, or not above every such entry
 * before it in its list, takes no part: a page counts once.  With all pages chosen the two calls mean the same.  Everything else
 * (values that are no numbers, rows that see nothing, limits of scores) as for mustdrop_cache4_attend; a probability always carries 16 bits
 * for MD_BF16.  Two calls on the same inputs, with lists and tables of the same width, give the same bits.  Errors likewise, and MD_ESHAPE for 2^23 or more tiles of 16 query heads or parts of them.
 * Lists of more than 1024 entries, and few long ones, are cut into parts, whose sums go through the workspace: its size is what calls with these
 * sizes and any table need at most, 4 (d + 2) bytes for each query head (of more than 16 to one: 16 at a time) and part; a call whose tokens go together has no parts and needs 256. */
size_t mustdrop_cache4_attend_chosen_workspace_bytes(int B, int N, int Hq, int H, int d, int budget, int page);

int mustdrop_cache4_attend_chosen(
    const void* q, md_dtype dtype, const void* cache, const int32_t* table, const int32_t* len, const int32_t* q_len, const uint8_t* keep,
    const int32_t* chosen, int B, int N, int Hq, int H, int d, int n_pages, int page, int max_pages, int budget, float softmax_scale,
    void* out, float* lse, const md_kv_layout* q_layout, const md_kv_layout* out_layout,
    void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MUSTDROP_H */
