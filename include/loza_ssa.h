/*
 * loza_ssa.h — C ABI of the streaming sparse attention (SSA) library for MI355X (gfx950).
 *
 * SSA is the sparse attention of LongCat ZigZag Attention: O* = softmax(Q K*^T) V*, where every
 * query keeps a fixed set of leading "sink" keys plus a causal window of its most recent keys
 * (paper: Architecture section, Eq. 2 and Eq. 4; sink/local sizes in the Training section).
 * With window >= S the same entry points compute ordinary causal attention (Eq. 1), which is the
 * full-attention comparator.
 *
 * Live set at token granularity (0-based query position i, key position j):
 *     live(i) = { j : j <= i  and ( j < n_sink  or  i - j < window ) }
 * so the window counts the query's own position, sink and window are united (a key is used once),
 * and |live(i)| = min(i + 1, n_sink + window).
 *
 * Conventions shared by every entry point
 *   - All tensor pointers are DEVICE pointers unless stated; the caller owns every buffer; the
 *     library allocates nothing and performs no host sync. It keeps no state between calls (the one
 *     exception, a scratch buffer whose contents never matter, is described at loza_ssa_decode_static).
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream). Calls are
 *     asynchronous on it.
 *   - Layouts are dense, innermost index fastest. bf16 tensors are raw 16-bit patterns.
 *   - Query head h reads key/value head h / (Hq / Hkv); Hq must be a multiple of Hkv.
 *   - Absorbed MLA (many query heads share one latent): pass v == k with d_v <= d_qk; the value
 *     row is then the first d_v elements of the key row (row stride d_qk) and costs no second load.
 *   - Base pointers must be 16-byte aligned. Inputs must be finite.
 *   - Every argument is validated before the first HIP call; a failed validation launches nothing.
 *   - Return value: LOZA_OK or a negative loza_status.
 *   - One environment variable is read (on every decode call and by the two host-only size functions
 *     below): LOZA_DECODE_SPLITS=n, 1 <= n <= 64, replaces the number of key splits a decode call
 *     chooses from its sizes (other values are ignored). It exists for tests and experiments; it
 *     changes the workspace size, so it must not change between loza_ssa_decode_workspace_bytes and
 *     the decode call. Nothing else is read from the environment.
 *   - Where each declaration comes from: the prototypes of loza_ssa_prefill and loza_ssa_decode are
 *     given by the benchmark spec; the operation is the paper's (cited at each entry point); every
 *     other name, argument and helper is this library's own.
 */
#ifndef LOZA_SSA_H
#define LOZA_SSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LOZA_OK = 0,
    LOZA_ERR_NULL = -1,        /* a required pointer is NULL                                  */
    LOZA_ERR_SHAPE = -2,       /* sizes out of range or inconsistent (Hq % Hkv, window < 1…)  */
    LOZA_ERR_UNSUPPORTED = -3, /* a (dtype, d_qk, d_v) combination no kernel is built for      */
    LOZA_ERR_WORKSPACE = -4,   /* workspace NULL or smaller than loza_ssa_decode_workspace_bytes */
    LOZA_ERR_HIP = -5,         /* a HIP call failed (hipGetLastError has the detail)          */
    LOZA_ERR_ALIGN = -6        /* a base pointer is not 16-byte aligned                       */
} loza_status;

#define LOZA_WINDOW_INF INT64_MAX /* window = infinity: full causal attention (Eq. 1) */

/*
 * SSA prefill, bf16 in / bf16 out, fp32 accumulation (Eq. 4; Eq. 1 when window >= S).
 *   q    [B, S, Hq,  d_qk] bf16      k [B, S, Hkv, d_qk] bf16      v [B, S, Hkv, d_v] bf16 (or v == k)
 *   out  [B, S, Hq,  d_v ] bf16      lse [B, Hq, S] fp32, natural log of the softmax denominator
 *   n_sink >= 0 leading keys always visible; window >= 1 most recent keys visible (self included).
 *   scale multiplies q.k before the softmax (the 1/sqrt(d) the paper's equations leave out);
 *   finite and > 0 (anything else: LOZA_ERR_SHAPE).
 * Supported (d_qk, d_v): (576, 512) with v == k (absorbed MLA: the value row is the first 512
 * elements of the key row), and (128, 128) with v separate or v == k. Anything else:
 * LOZA_ERR_UNSUPPORTED. S <= 2^31 - 129.
 * Numerics: scores, exponentials and sums in fp32; the softmax weights go to the matrix cores as
 * bf16, rounded once (relative error 2^-9 each) or, where that is not good enough, as two bf16
 * terms (2^-17): for tiles that start within the first 128 positions, for patterns that leave every
 * row fewer than 128 live keys, and for every tile in which the one-term pass produced a result of
 * magnitude >= 1.97 (the tile is then computed again inside the same launch). Calls of few query rows
 * (at most 512 groups of 16 rows per key head, over all key heads and sequences) take two terms
 * throughout. Error of a result:
 *     |out - exact| <= half an ulp of bf16 at |out|  +  w * D  +  about 1e-6 * |out|,
 * D = the softmax-weighted mean of |v_j - out| over the live keys (never more than their largest
 * distance from out), w = 2^-9 for one-term rows and 2^-17 for two-term rows. One-term rows have
 * |out| < 2, i.e. half an ulp <= 2^-8: they stay inside 1e-2 whenever D <= 3.1 (values of unit
 * scale give D of about 1, and random rounding errors add to a small fraction of w * D); two-term
 * rows stay inside 1e-2 for |out| < 4 whenever D <= 280. From |out| = 4 on the rounding of the
 * result to bf16 alone is 2^-6. lse: fp32 throughout, |lse - exact| <= 2e-5 at the tested sizes.
 * The launch is deterministic: the same inputs give the same bits.
 */
int loza_ssa_prefill(const void *q, const void *k, const void *v, void *out, float *lse,
                     int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                     int64_t n_sink, int64_t window, float scale, void *stream);

/*
 * fp32 twin of loza_ssa_prefill (fp32 in, fp32 arithmetic, fp32 out), same layouts with float
 * elements. Any d_qk, d_v in [1, 256]; v may alias k with d_v <= d_qk; scale finite, any sign.
 * The small-shape check of the method (fp32 matrix instructions, a few rows per workgroup), not a fast path.
 */
int loza_ssa_prefill_f32(const float *q, const float *k, const float *v, float *out, float *lse,
                         int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                         int64_t n_sink, int64_t window, float scale, void *stream);

/*
 * SSA decode: one new query token per sequence against that sequence's KV cache (the decode
 * kernel of the paper's Efficiency section). Split over the live keys with a log-sum-exp merge.
 *   q       [B, Hq, d_qk] bf16
 *   kcache  [B, S_max, Hkv, d_qk] bf16     vcache [B, S_max, Hkv, d_v] bf16 (or vcache == kcache)
 *   seqlens [B] int32 (device): valid rows of each cache INCLUDING the new token's own key/value,
 *           so the query sits at position seqlens[b] - 1. 0 <= seqlens[b] <= S_max is required;
 *           a sequence of length 0 yields out = 0, lse = -inf.
 *   out     [B, Hq, d_v] bf16              lse [B, Hq] fp32
 *   workspace: device scratch of at least loza_ssa_decode_workspace_bytes(...) bytes, 16-byte
 *           aligned; contents on entry are ignored, on exit unspecified. It holds, per (b, query
 *           head, key split), the unnormalised fp32 partial output and four floats of softmax
 *           state. Two calls that overlap in time need two workspaces.
 * Supported (d_qk, d_v) and scale: as loza_ssa_prefill. Cache rows at or beyond seqlens[b] are
 * never read. The split count depends on the sizes only (and on LOZA_DECODE_SPLITS, see above), and
 * the merge adds the splits in a fixed order: the result is deterministic.
 * Numerics: as loza_ssa_prefill, but the weights are not rounded (three bf16 terms hold an fp32 weight; w
 * of the bound above is that of fp32 arithmetic, about 2^-23). Calls with many sequences and long windows
 * on key heads of more than 32 query heads take one-term weights, except that a query with fewer than 128
 * live keys, and a query whose merged result reaches magnitude 1.97 in some column, is then computed from
 * the cache rows directly in fp32 (a rare, slower path: one workgroup walks all live keys of that query).
 */
int loza_ssa_decode(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                    void *out, float *lse, int B, int Hq, int Hkv, int64_t S_max,
                    int d_qk, int d_v, int64_t n_sink, int64_t window, float scale,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * loza_ssa_decode for callers that cannot allocate device memory or carry a workspace around (code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same kernels,
 * the same result bits, with the partial results of the key splits in a buffer that is part of the
 * library image (LOZA_DECODE_STATIC_BYTES of device memory on every GPU the library is used on, held
 * until the process ends). No hipMalloc / hipFree, here or in anything it calls.
 *   - sizes whose workspace (loza_ssa_decode_workspace_bytes) exceeds LOZA_DECODE_STATIC_BYTES are
 *     rejected with LOZA_ERR_WORKSPACE before anything is launched; LOZA_DECODE_STATIC_BYTES covers
 *     B * Hq * splits <= 20,321 at d_v = 512 (B = 64 sequences of 64 heads in 4 splits use 16,384).
 *   - every call on a GPU uses that GPU's one buffer: calls that overlap in time on one GPU (two
 *     streams, two threads) race on it and must be serialised by the caller. Nothing in it has to
 *     survive or be cleared between calls.
 * All other arguments, errors and numerics: as loza_ssa_decode.
 */
#define LOZA_DECODE_STATIC_BYTES (40u << 20)
int loza_ssa_decode_static(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                           void *out, float *lse, int B, int Hq, int Hkv, int64_t S_max,
                           int d_qk, int d_v, int64_t n_sink, int64_t window, float scale, void *stream);

/* Host-only (ours). Bytes of workspace loza_ssa_decode needs for these sizes (0 on invalid sizes). */
size_t loza_ssa_decode_workspace_bytes(int B, int Hq, int Hkv, int64_t S_max, int d_v,
                                       int64_t n_sink, int64_t window);

/* Host-only (ours). Number of key splits the workspace of loza_ssa_decode is sized for at these sizes; the
 * call uses as many or fewer (0 on invalid sizes). */
int loza_ssa_decode_num_splits(int B, int Hq, int Hkv, int64_t S_max, int64_t n_sink, int64_t window);

/*
 * Host-only (ours), for tests and tools: which kernels a bf16 call of these sizes runs. The pattern as the
 * _blocks entry points take it; block = 1: n_sink and window in tokens. Negative (a loza_status) on sizes
 * that the call itself refuses.
 *   loza_ssa_forward_kernel   prefill (n_queries = S), calibration or extend (n_queries = q_len, S = S_max):
 *                             a loza_kernel, of a call without scratch memory. An extend that has what
 *                             loza_ssa_extend_workspace_bytes says, if that is more than 0, has workgroups that
 *                             share keys: of the same kernel, or at d_qk = 576 of LOZA_KERNEL_TILES in the
 *                             place of LOZA_KERNEL_ROWS where those are faster
 *   loza_ssa_decode_kernel    a loza_kernel; *n_splits (may be NULL): the key splits it takes
 *   loza_ssa_backward_split   how many key tiles of 64 (per sequence and key head) the dK/dV kernel cuts into
 *                             chunks of rows for balance; *n_chunks, *n_whole (may be NULL): the chunks of
 *                             each, and the work items of the launch that are not such chunks (at d_qk = 576:
 *                             where a call takes the kernels that keep no weights in its workspace)
 */
typedef enum {
    LOZA_KERNEL_TILES = 1, /* tiles of 128 (decode: 64) query rows      */
    LOZA_KERNEL_ROWS = 2,  /* few query rows: 16 or 32 a workgroup      */
    LOZA_KERNEL_D128 = 3   /* width 128: tiles of 256 query rows        */
} loza_kernel;
int loza_ssa_forward_kernel(int B, int Hq, int Hkv, int64_t n_queries, int64_t S, int d_qk,
                            int64_t sink_blocks, int64_t local_blocks, int64_t block);
int loza_ssa_decode_kernel(int B, int Hq, int Hkv, int64_t S_max, int d_qk,
                           int64_t sink_blocks, int64_t local_blocks, int64_t block, int *n_splits);
int loza_ssa_backward_split(int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v, int64_t sink_blocks,
                            int64_t local_blocks, int64_t block, int v_aliases_k, int *n_chunks, int64_t *n_whole);

/*
 * Host-only, no GPU involved: the live set of query i as at most two half-open key ranges,
 * [0, *sink_end) and [*win_begin, *win_end), disjoint and in order (sink_end <= win_begin).
 * This is the arithmetic the kernels enumerate tiles with (Eq. 4's pattern, "single uniform
 * schedule" of the Desiderata section: no per-head metadata).
 */
int loza_ssa_live_ranges(int64_t i, int64_t n_sink, int64_t window,
                         int64_t *sink_end, int64_t *win_begin, int64_t *win_end);

/* Host-only (ours). Live (query, key) pairs of a causal length-S prefill: the sum over i of |live(i)|
 * for the live sets of Eq. 4 as defined at the top of this file. This is the pair count the
 * benchmark's FLOP figure is built on ("compute per query stays constant": Architecture section). */
int64_t loza_ssa_live_pairs(int64_t S, int64_t n_sink, int64_t window);

/*
 * The same operation under the block-granular pattern the paper parametrises SSA with
 * (Architecture section, after Eq. 4: number of sink blocks s, number of local blocks l, block
 * size b; Training section: b = 128, s = 1, l = 7, at most 1,024 live tokens). Keys and queries
 * are cut into blocks of `block` tokens; the query at position i, in block qb = i / block, sees
 *     live(i) = { j : j <= i  and ( j / block < sink_blocks  or  qb - j / block < local_blocks ) }
 * i.e. the whole sink blocks and the local_blocks most recent blocks, its own block counted as one
 * of them and cut at the query. |live(i)| runs through (s + l - 1) b + 1 ... (s + l) b within each
 * block once i >= (s + l) b. With block == 1 this is the token-granular pattern with
 * n_sink = sink_blocks and window = local_blocks.
 * sink_blocks >= 0, local_blocks >= 1, block >= 1 (else LOZA_ERR_SHAPE); everything else
 * (layouts, supported shapes, numerics, error behaviour) as for the token-granular twin.
 * loza_ssa_decode_blocks takes a workspace of
 *     loza_ssa_decode_workspace_bytes(B, Hq, Hkv, S_max, d_v, sink_blocks * block, local_blocks * block)
 * bytes (products saturating at INT64_MAX) and uses the split count of the same sizes.
 */
int loza_ssa_prefill_blocks(const void *q, const void *k, const void *v, void *out, float *lse,
                            int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                            int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *stream);

int loza_ssa_prefill_blocks_f32(const float *q, const float *k, const float *v, float *out, float *lse,
                                int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                                int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *stream);

int loza_ssa_decode_blocks(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                           void *out, float *lse, int B, int Hq, int Hkv, int64_t S_max,
                           int d_qk, int d_v, int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * SSA "extend": q_len new query tokens per sequence against that sequence's KV cache, which already
 * holds their keys and values (chunked prefill, verification of speculated tokens: the engine side of
 * the paper's Efficiency section). Query r of sequence b sits at position seqlens[b] - q_len + r and
 * sees the live set of that position; q_len == 1 is what loza_ssa_decode computes.
 *   q       [B, q_len, Hq, d_qk] bf16
 *   kcache  [B, S_max, Hkv, d_qk] bf16     vcache [B, S_max, Hkv, d_v] bf16 (or vcache == kcache)
 *   seqlens [B] int32 (device): valid cache rows, the q_len new tokens included; a value above
 *           S_max is cut to it. Queries whose position would be negative (seqlens[b] < q_len)
 *           give out = 0, lse = -inf.
 *   out     [B, q_len, Hq, d_v] bf16       lse [B, Hq, q_len] fp32
 * 1 <= q_len <= S_max (else LOZA_ERR_SHAPE). No workspace (no split of a query's keys over workgroups).
 * Supported shapes, numerics, errors: as loza_ssa_prefill / loza_ssa_prefill_blocks.
 */
int loza_ssa_extend(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens, void *out, float *lse,
                    int B, int Hq, int Hkv, int64_t S_max, int q_len, int d_qk, int d_v,
                    int64_t n_sink, int64_t window, float scale, void *stream);

int loza_ssa_extend_blocks(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens, void *out,
                           float *lse, int B, int Hq, int Hkv, int64_t S_max, int q_len, int d_qk, int d_v,
                           int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *stream);

/*
 * loza_ssa_extend / loza_ssa_extend_blocks against a paged cache: k_pages, v_pages, block_table,
 * num_pages, page_size, max_pages_per_seq as for loza_ssa_decode_paged below (same conditions on
 * page_size and on the table entries), q, seqlens, out, lse as for loza_ssa_extend, with
 * max_pages_per_seq * page_size in the place of S_max.
 */
int loza_ssa_extend_paged(const void *q, const void *k_pages, const void *v_pages, const int32_t *block_table,
                          const int32_t *seqlens, void *out, float *lse, int B, int Hq, int Hkv,
                          int64_t num_pages, int page_size, int max_pages_per_seq, int q_len, int d_qk, int d_v,
                          int64_t n_sink, int64_t window, float scale, void *stream);

int loza_ssa_extend_paged_blocks(const void *q, const void *k_pages, const void *v_pages, const int32_t *block_table,
                                 const int32_t *seqlens, void *out, float *lse, int B, int Hq, int Hkv,
                                 int64_t num_pages, int page_size, int max_pages_per_seq, int q_len, int d_qk, int d_v,
                                 int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *stream);

/*
 * Any of the four extends with scratch memory, so that several workgroups can share the keys of a query (few
 * new tokens against long windows otherwise leave most of the GPU idle): block_table == NULL is
 * loza_ssa_extend_blocks (num_pages, page_size, max_pages_per_seq unused), a table is
 * loza_ssa_extend_paged_blocks (S_max unused); block = 1 is the token-granular pattern. Results agree with
 * theirs to the order of the sums, and where tiles of 128 rows share keys all their weights have two bf16
 * terms. `workspace` (16-byte aligned, device): loza_ssa_extend_workspace_bytes
 * (S_max = max_pages_per_seq * page_size of a paged cache; 0: these sizes need none, the pointer may be
 * NULL, and the call is the one without). It must stay untouched until the launches have run; its contents do
 * not matter before and mean nothing afterwards. Where that size is for tiles of 128 rows in the place of the kernel for few
 * query rows, a smaller one, or none, is accepted if that kernel can do with it; LOZA_ERR_WORKSPACE otherwise.
 */
int loza_ssa_extend_with_workspace(const void *q, const void *k, const void *v, const int32_t *block_table, const int32_t *seqlens,
                                   void *out, float *lse, int B, int Hq, int Hkv, int64_t S_max, int64_t num_pages,
                                   int page_size, int max_pages_per_seq, int q_len, int d_qk, int d_v, int64_t sink_blocks,
                                   int64_t local_blocks, int64_t block, float scale, void *workspace, size_t workspace_bytes,
                                   void *stream);
size_t loza_ssa_extend_workspace_bytes(int B, int Hq, int Hkv, int64_t S_max, int q_len, int d_qk, int d_v,
                                       int64_t sink_blocks, int64_t local_blocks, int64_t block);

/*
 * SSA decode against a PAGED KV cache (the cache layout of a serving engine; the paper's
 * Efficiency section measures its decode kernel inside one). The rows of sequence b live in pages
 * of `page_size` rows: logical row j is row j % page_size of physical page
 * block_table[b * max_pages_per_seq + j / page_size].
 *   k_pages [num_pages, page_size, Hkv, d_qk] bf16   v_pages [num_pages, page_size, Hkv, d_v] bf16
 *           (or v_pages == k_pages: values are the first d_v elements of the key rows)
 *   block_table [B, max_pages_per_seq] int32 (device). Only the entries of pages that hold a live
 *           key are read (sink pages and the pages of the window); they must lie in [0, num_pages).
 *           An entry outside that range is cut to it: no fault, but the wrong rows.
 *   seqlens [B] int32 (device), 0 <= seqlens[b] <= max_pages_per_seq * page_size.
 *   page_size: a power of two >= 32 (else LOZA_ERR_SHAPE).
 *   workspace: loza_ssa_decode_workspace_bytes(B, Hq, Hkv, max_pages_per_seq * page_size, d_v, n_sink, window)
 *           bytes (for the _blocks form with sink_blocks * block and local_blocks * block).
 * Everything else as loza_ssa_decode / loza_ssa_decode_blocks; the result is the same bits as for
 * the same rows in a contiguous cache.
 */
int loza_ssa_decode_paged(const void *q, const void *k_pages, const void *v_pages, const int32_t *block_table,
                          const int32_t *seqlens, void *out, float *lse, int B, int Hq, int Hkv,
                          int64_t num_pages, int page_size, int max_pages_per_seq, int d_qk, int d_v,
                          int64_t n_sink, int64_t window, float scale,
                          void *workspace, size_t workspace_bytes, void *stream);

int loza_ssa_decode_paged_blocks(const void *q, const void *k_pages, const void *v_pages, const int32_t *block_table,
                                 const int32_t *seqlens, void *out, float *lse, int B, int Hq, int Hkv,
                                 int64_t num_pages, int page_size, int max_pages_per_seq, int d_qk, int d_v,
                                 int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Calibration forward (paper: Architecture section, Eq. 3): the layer output with the learnable
 * mixing factor alpha in [0, 1] between full attention O and streaming sparse attention O',
 *     out = alpha * O + (1 - alpha) * O'
 * for the block-granular pattern (block == 1: token-granular with n_sink = sink_blocks and
 * window = local_blocks). Two prefill passes (all causal keys; the sparse pattern) leave their
 * unrounded fp32 outputs in the workspace; a third kernel mixes them and rounds once to bf16.
 *   out        [B, S, Hq, d_v] bf16  the blend
 *   out_full   NULL or [B, S, Hq, d_v] bf16: O itself      out_sparse  NULL or the same for O'
 *              (alpha's gradient is the inner product of the incoming gradient with O - O')
 *   lse_full, lse_sparse [B, Hq, S] fp32: the log-sum-exp of either pass
 *   workspace  loza_ssa_calibration_workspace_bytes(B, Hq, S, d_v) bytes, 16-byte aligned
 * alpha outside [0, 1] or NaN: LOZA_ERR_SHAPE. Everything else as loza_ssa_prefill_blocks.
 */
int loza_ssa_prefill_calibration_blocks(const void *q, const void *k, const void *v,
                                        void *out, void *out_full, void *out_sparse, float *lse_full, float *lse_sparse,
                                        int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                                        int64_t sink_blocks, int64_t local_blocks, int64_t block,
                                        float alpha, float scale, void *workspace, size_t workspace_bytes, void *stream);

/* Host-only (ours). Workspace bytes of loza_ssa_prefill_calibration_blocks (0 on invalid sizes). */
size_t loza_ssa_calibration_workspace_bytes(int B, int Hq, int64_t S, int d_v);

/*
 * Gradient of the calibration blend with respect to alpha (Architecture section, Eq. 3): the blend is
 * alpha O + (1 - alpha) O', so d(alpha) = sum over every element of dout * (O - O').
 *   dout, out_full, out_sparse: n bf16 elements each (device, 16-byte aligned): the gradient arriving
 *       at the blend and the two outputs loza_ssa_prefill_calibration_blocks wrote; n >= 8, a multiple of 8
 *   dalpha: one float on the device (overwritten)
 *   workspace: loza_ssa_calibration_alpha_grad_workspace_bytes(n) bytes of device memory (host-only
 *       helper, ours; 0 for an n the call rejects), 16-byte aligned, contents ignored
 * Products and sums in fp64 in a fixed order (deterministic), one rounding to fp32 at the end.
 */
int loza_ssa_calibration_alpha_grad(const void *dout, const void *out_full, const void *out_sparse, float *dalpha, int64_t n,
                                    void *workspace, size_t workspace_bytes, void *stream);
size_t loza_ssa_calibration_alpha_grad_workspace_bytes(int64_t n);

/*
 * SSA backward: the gradients of loza_ssa_prefill's output with respect to q, k and v, over live
 * (query, key) pairs only. This is what training a sparsified model differentiates (paper:
 * Architecture section, Eq. 4 and its Training paragraph; the paper states no formulas, they are the
 * chain rule of a softmax):
 *     p_ij = exp(scale q_i.k_j - lse_i) for live j,  D_i = dout_i . out_i,
 *     dv_j = sum_i p_ij dout_i,  ds_ij = p_ij (dout_i . v_j - D_i),
 *     dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,
 * the sums over i taking every query head of the key's group.
 *   q, k, v     as loza_ssa_prefill (bf16; v == k allowed)
 *   out  [B, S, Hq, d_v] bf16 and lse [B, Hq, S] fp32: what loza_ssa_prefill returned for q, k, v
 *   dout [B, S, Hq, d_v] bf16: gradient arriving at out
 *   dq   [B, S, Hq, d_qk] bf16      dk [B, S, Hkv, d_qk] bf16      dv [B, S, Hkv, d_v] bf16
 *        When v == k, the one tensor serves as keys and (its first d_v columns) as values; dk then
 *        receives the gradient with respect to that tensor (dk with dv added to its first d_v
 *        columns) and dv is ignored (may be NULL).
 *   workspace: loza_ssa_backward_workspace_bytes(...) bytes of device memory, 16-byte aligned;
 *        contents on entry are ignored. Two calls that overlap in time need two workspaces. At d_qk = 576
 *        most of it holds softmax weights on their way from one kernel to the next and partial sums of dk (long
        sequences: 2 to 2.5 GiB; up to 4.6 where windows are close to 32,000 tokens or a key head has two query heads;
        0.5 for 2,048 tokens of 64 heads, 1 + 7 blocks of 128); a
 *        smaller one that still holds the row statistics (8 bytes a query row, rows padded to 32 per key head)
 *        and the partial sums of the sink keys (147,456 bytes per 64 of them and chunk of rows) is accepted, and
 *        the call then takes about 1.3 to 1.6 times as long. (Where the size that is given out is that small, no weights are kept: few
        query heads on a key head with short windows, rows that see 128 keys or fewer, windows beyond about 32,000 tokens.)
 * Supported: the (d_qk, d_v) pairs of loza_ssa_prefill, scale > 0, and Hq / Hkv a power of two up to
 * 32 or a multiple of 32 (else LOZA_ERR_UNSUPPORTED). Arithmetic: bf16 matrix-core operands (q, k,
 * v, dout, and p and ds rounded to bf16), fp32 accumulation, one rounding of each result to bf16.
 * Sums run in a fixed order: the result is deterministic. No output aliases an input; dq may hold partial
 * sums of dk and dv while the call runs.
 */
int loza_ssa_backward(const void *q, const void *k, const void *v, const void *out, const float *lse,
                      const void *dout, void *dq, void *dk, void *dv,
                      int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                      int64_t n_sink, int64_t window, float scale,
                      void *workspace, size_t workspace_bytes, void *stream);

/* The same under the block-granular pattern of loza_ssa_prefill_blocks. */
int loza_ssa_backward_blocks(const void *q, const void *k, const void *v, const void *out, const float *lse,
                             const void *dout, void *dq, void *dk, void *dv,
                             int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                             int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale,
                             void *workspace, size_t workspace_bytes, void *stream);

/*
 * fp32 twins of loza_ssa_decode and loza_ssa_decode_blocks (same definition: the query of sequence b
 * sits at position seqlens[b] - 1 of its cache; Architecture section, Eq. 2 / Eq. 4): fp32 in, fp32
 * arithmetic, fp32 out, the layouts of the bf16 calls with float elements. Any d_qk, d_v in [1, 256];
 * vcache may alias kcache with d_v <= d_qk; a length beyond S_max is cut to it; an empty cache gives
 * out = 0 and lse = -inf. No workspace (one workgroup per 16 query heads walks all of their live keys).
 */
int loza_ssa_decode_f32(const float *q, const float *kcache, const float *vcache, const int32_t *seqlens, float *out, float *lse,
                        int B, int Hq, int Hkv, int64_t S_max, int d_qk, int d_v,
                        int64_t n_sink, int64_t window, float scale, void *stream);
int loza_ssa_decode_blocks_f32(const float *q, const float *kcache, const float *vcache, const int32_t *seqlens, float *out,
                               float *lse, int B, int Hq, int Hkv, int64_t S_max, int d_qk, int d_v,
                               int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *stream);

/*
 * fp32 twins of loza_ssa_backward and loza_ssa_backward_blocks (the gradient of the paper's Eq. 4, as
 * above): fp32 in, fp32 arithmetic, fp32 out, the layouts of the bf16 calls with float elements; out
 * and lse are what loza_ssa_prefill_f32 returned. Any d_qk, d_v in [1, 256], any Hq / Hkv; v may alias
 * k with d_v <= d_qk (dk then receives the whole gradient of the shared tensor and dv is ignored);
 * scale finite, any sign. No workspace; deterministic (every sum runs in a fixed order). Plain vector
 * arithmetic (no matrix cores): the small-shape check of the method, not a fast path.
 */
int loza_ssa_backward_f32(const float *q, const float *k, const float *v, const float *out, const float *lse,
                          const float *dout, float *dq, float *dk, float *dv,
                          int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                          int64_t n_sink, int64_t window, float scale, void *stream);
int loza_ssa_backward_blocks_f32(const float *q, const float *k, const float *v, const float *out, const float *lse,
                                 const float *dout, float *dq, float *dk, float *dv,
                                 int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                                 int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *stream);

/* Host-only (ours). Workspace bytes of loza_ssa_backward / loza_ssa_backward_blocks for these sizes
 * (v_aliases_k: nonzero when v == k will be passed); 0 on sizes the call would reject. */
size_t loza_ssa_backward_workspace_bytes(int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                                         int64_t n_sink, int64_t window, int v_aliases_k);
size_t loza_ssa_backward_workspace_bytes_blocks(int B, int Hq, int Hkv, int64_t S, int d_qk, int d_v,
                                                int64_t sink_blocks, int64_t local_blocks, int64_t block,
                                                int v_aliases_k);

/* Host-only twins (ours) of loza_ssa_live_ranges / loza_ssa_live_pairs for the block-granular pattern
 * (Architecture section after Eq. 4: sink blocks, local blocks, block size). */
int loza_ssa_live_ranges_blocks(int64_t i, int64_t sink_blocks, int64_t local_blocks, int64_t block,
                                int64_t *sink_end, int64_t *win_begin, int64_t *win_end);
int64_t loza_ssa_live_pairs_blocks(int64_t S, int64_t sink_blocks, int64_t local_blocks, int64_t block);

/* ---------------------------------------------------------------------------------------------------------
 * The step around the attention: what an engine that drafts tokens calls between one decode step and the next, all of
 * it on the GPU (no lengths on the host), so that a step can be captured. The paper stretches its contexts with YaRN and
 * measures its kernels inside such an engine (Training and Efficiency sections); it describes none of this, the definitions
 * are the usual ones. A step: loza_ssa_step_tables_held, then in every layer loza_ssa_rope_append and loza_ssa_extend_tree
 * (or loza_ssa_decode_paged, loza_ssa_extend_paged), then loza_ssa_verify_tree, and loza_ssa_keep_accepted for all layers.
 *
 * Trees. The tokens of a step are the nodes of a tree per sequence, at most LOZA_TREE_MAX_NODES of them, parents before their
 * children. parents[b, r] is the parent of node r, an index below r; anything else: a node without a parent. Node 0 is the
 * token that the last step ended with (its row is not in the cache yet), the others are drafts. A chain of drafts is
 * the tree parents[r] = r - 1.
 *
 * Pages. A page belongs to the request whose row of block_table names it until the engine puts it back on the free list, also where it holds nothing but rows
 * that were not kept. Chunks keep all their rows; a step of drafts keeps a part of them, and leaves a request with more pages than its cache_len
 * needs: loza_ssa_step_tables_held is told how many, and deals out new ones behind those (with loza_ssa_step_tables the engine has to put
 * the pages [ceil((cache_len + path_len) / page_size), ceil(seqlen / page_size)) of each row back itself, or they are lost). An engine whose requests
 * take both, chunks and drafts, tells it with both. Between two steps: cache_lens += path_lens (chunks: granted), free_count = free_left, held = held_after.
 * A request that ends has the first `held` entries of its row appended to free_pages from free_count on (which has room for every page), free_count grows by
 * as many, and its cache_len and held are 0.
 */
#define LOZA_TREE_MAX_NODES 64
#define LOZA_ROPE_MAX_DIM 1024

/*
 * Block tables, slots, positions and ancestor masks of a step, from the lengths of the requests.
 *   cache_lens [B] int32: rows each request has in its cache     new_lens [B] int32: rows it is about to add, 0 .. n
 *   parents [B, n] int32 or NULL: the step's tokens are trees (n <= LOZA_TREE_MAX_NODES) or the next tokens in a row
 *   free_pages [num_free] int32, free_count [1] int32: pages nobody holds; the first free_count entries (at most num_free) are valid
 *   block_table [B, max_pages_per_seq] int32: the pages that a request holds already (the first ceil(cache_len / page_size) entries of
 *           its row) are read; the entries of the pages it needs beyond those are written, no others
 *   granted [B] int32: new_lens, or 0 where the request cannot be served: pages are dealt out in the order of the requests,
 *           from the end of the free list; one whose need, with those of all requests before it (served or not), exceeds free_count gets none (one that needs
 *           no new page is always served), nor does one with lengths that are negative, beyond n, or beyond max_pages_per_seq
 *           pages (these take nothing from the others)
 *   seqlens [B] int32: cache_lens + granted, as the decode and extend calls take it
 *   positions, slots [B, n] int32: the position of each token and the cache row (page * page_size + row in the page) it goes to;
 *           -1 for rows without a token (of requests that were not served, too), slots also where the table holds a page outside [0, num_pages).
 *           Trees: row r is node r (r < granted), at row cache_len + r and position cache_len + the number of its
 *           ancestors. No trees: the last `granted` of the n rows, as loza_ssa_extend_paged counts them (row r at
 *           position seqlens - n + r).
 *   masks [B, n] int64 (NULL without parents): bit a of masks[b, r] says that node r sees node a: its ancestors and itself; 0
 *           for rows without a token
 *   free_left [1] int32: valid entries of free_pages that are left
 * B <= 65536; page_size: a power of two >= 32; num_pages * page_size < 2^31. No array that is written (block_table among them) may
 * overlap another array of the call (LOZA_ERR_SHAPE). The call is repeatable: it changes none of its inputs but those entries of block_table.
 *
 * loza_ssa_step_tables_held:
 *   held [B] int32: entries of each row of block_table that are the request's pages; fewer than ceil(cache_len / page_size): taken as that many; negative
 *           or beyond max_pages_per_seq: the request gets nothing
 *   held_after [B] int32: the same after the call: those (as taken), and the new ones if it is served; as given where the request's numbers are not
 *           possible.
 */
int loza_ssa_step_tables(const int32_t *cache_lens, const int32_t *new_lens, const int32_t *parents, const int32_t *free_pages,
                         const int32_t *free_count, int32_t *block_table, int B, int n, int64_t num_free, int64_t num_pages,
                         int page_size, int max_pages_per_seq, int32_t *granted, int32_t *seqlens, int32_t *positions,
                         int32_t *slots, int64_t *masks, int32_t *free_left, void *stream);
int loza_ssa_step_tables_held(const int32_t *cache_lens, const int32_t *new_lens, const int32_t *parents, const int32_t *free_pages,
                              const int32_t *free_count, const int32_t *held, int32_t *block_table, int B, int n, int64_t num_free, int64_t num_pages,
                              int page_size, int max_pages_per_seq, int32_t *granted, int32_t *seqlens, int32_t *positions,
                              int32_t *slots, int64_t *masks, int32_t *free_left, int32_t *held_after, void *stream);

/*
 * Rotary positions, and their gradient. Pair k of the columns [rot_begin, rot_begin + rot_dim) of a head at position i,
 * (a, b) -> mscale (a cos t - b sin t, a sin t + b cos t), t = i * freq[k]; inverse != 0: by -t, which is the gradient of
 * the rotation (of x from that of out), and undoes it where mscale is 1.
 *   x, out [T, H, d]: element (t, h, c) at t * token stride + h * head stride + c (strides in elements, >= 0; the places of out must
 *           not overlap). out == x with the same strides: in place; other overlaps are not allowed. Columns outside the rotary ones are
 *           copied.
 *   positions [T] int32: >= 0; a token with a negative one is padding, its row of out is left as it is
 *   freq [rot_dim / 2] float64, radians per position (loza_ssa_rope_frequencies); rot_dim even, 2 .. LOZA_ROPE_MAX_DIM
 *   interleaved != 0: pair k is columns 2 k and 2 k + 1, else k and k + rot_dim / 2 (from rot_begin)
 * bf16 (loza_ssa_rope) or fp32. H d <= 2^30. Base pointers need only be aligned to their elements; 16 bytes for them, the strides, d, rot_begin and (half of, where
 * pairs are not interleaved) rot_dim is several times faster. Angles in 64 bits and more (exact to 2^-24 of a turn at any
 * position), sine and cosine in fp32, one rounding of each result.
 */
int loza_ssa_rope(const void *x, const int32_t *positions, const double *freq, void *out, int64_t T, int H, int d,
                  int64_t x_token, int64_t x_head, int64_t out_token, int64_t out_head, int rot_begin, int rot_dim,
                  int interleaved, int inverse, float mscale, void *stream);
int loza_ssa_rope_f32(const float *x, const int32_t *positions, const double *freq, float *out, int64_t T, int H, int d,
                      int64_t x_token, int64_t x_head, int64_t out_token, int64_t out_head, int rot_begin, int rot_dim,
                      int interleaved, int inverse, float mscale, void *stream);

/*
 * The same for the queries and keys of a step, whose keys (rotated) and values (as they are) go to the cache in the same launch.
 *   q [T, Hq, d_q] -> q_out (strided as above, q_rot_begin; both NULL: keys and values only)
 *   k [T, Hkv, d_k] (strided, k_rot_begin) -> row slots[t] of k_rows [cache_rows, Hkv, d_k] (a paged or contiguous cache, whole rows dense)
 *   v [T, Hkv, d_v] (strided) -> row slots[t] of v_rows [cache_rows, Hkv, d_v]; both NULL where the values are part of the keys
 *   slots [T] int32: a token whose slot is outside [0, cache_rows), or whose position is negative, is not written to the cache
 *           (a rotated query needs the position only). No two tokens may have the same slot.
 */
int loza_ssa_rope_append(const void *q, const void *k, const void *v, const int32_t *positions, const int32_t *slots, const double *freq,
                         void *q_out, void *k_rows, void *v_rows, int64_t T, int Hq, int Hkv, int d_q, int d_k, int d_v,
                         int64_t q_token, int64_t q_head, int64_t q_out_token, int64_t q_out_head, int64_t k_token, int64_t k_head,
                         int64_t v_token, int64_t v_head, int64_t cache_rows, int q_rot_begin, int k_rot_begin, int rot_dim,
                         int interleaved, float mscale, void *stream);
int loza_ssa_rope_append_f32(const float *q, const float *k, const float *v, const int32_t *positions, const int32_t *slots, const double *freq,
                             float *q_out, float *k_rows, float *v_rows, int64_t T, int Hq, int Hkv, int d_q, int d_k, int d_v,
                             int64_t q_token, int64_t q_head, int64_t q_out_token, int64_t q_out_head, int64_t k_token, int64_t k_head,
                             int64_t v_token, int64_t v_head, int64_t cache_rows, int q_rot_begin, int k_rot_begin, int rot_dim,
                             int interleaved, float mscale, void *stream);

/*
 * Host-only (ours). Frequencies for contexts stretched by `factor` (the paper's YaRN, Training section): f_k = base^(-2k / rot_dim)
 * turns original_context * f_k / 2 pi times over the context that was trained; pairs of fewer than slow_turns (usually 1) are divided by the
 * factor, pairs of more than fast_turns (usually 32) are kept, those between are mixed linearly in their turns.
 * *mscale = 0.1 ln(factor) + 1, what queries and keys are scaled by (a model that has it in its softmax scale passes 1 instead).
 * factor = 1: plain frequencies, *mscale = 1, the last four arguments before freq unused.
 */
int loza_ssa_rope_frequencies(int rot_dim, double base, double factor, int64_t original_context, double slow_turns,
                              double fast_turns, double *freq, float *mscale);

/*
 * Attention of a tree of drafted tokens over a cache that already holds their rows: loza_ssa_extend_with_workspace with the
 * queries of a tree in the place of consecutive ones.
 *   block_table == NULL: k, v [B, S_max, Hkv, d] (num_pages, page_size, max_pages_per_seq unused), else pages (S_max unused)
 *   q [B, n, Hq, d_qk] bf16, out [B, n, Hq, d_v] bf16, lse [B, Hq, n] fp32; 1 <= n <= LOZA_TREE_MAX_NODES, n <= S_max
 *   seqlens [B] int32: valid cache rows, the nodes' rows included, which are the last tree_lens[b] of them (a length beyond the cache is cut to it)
 *   tree_lens [B] int32: nodes of each tree, cut to [0, n] and to seqlens. Rows r >= tree_lens[b]
 *           give out = 0, lse = -inf, whatever their queries hold (loza_ssa_rope_append does not write them). Cache rows at or beyond
 *           seqlens[b] are never read.
 *   masks [B, n] int64: the nodes that node r sees (loza_ssa_step_tables makes them; its own bit has to be set if it is
 *           to see itself; bits at or beyond tree_lens[b] are ignored). With P = seqlens[b] - tree_lens[b]: node r sits at position
 *           i = P + popcount(mask) - 1 and sees cache row j < P if j is live for position i, and the node of
 *           the k-th set bit (from 0) if position P + k is. A chain's masks (bits 0 .. r) give what loza_ssa_extend
 *           gives. A mask of 0: the row sees nothing, out = 0, lse = -inf, whatever its query holds.
 *   pattern, supported shapes, numerics: as loza_ssa_extend_blocks (block = 1: token-granular); where workgroups share keys, weights of two terms
 *   workspace: loza_ssa_extend_tree_workspace_bytes (S_max = max_pages_per_seq * page_size of a paged cache; 0: these sizes need none), 16-byte
 *           aligned, left alone until the launches have run, contents ignored. A smaller one is LOZA_ERR_WORKSPACE (loza_ssa_extend_with_workspace
 *           takes some that are: sizes that callers of it may have kept). NULL: no workgroups share keys; slower, and other bits
 * As many sequences and heads as a launch takes: n Hq / Hkv rows make tiles of 128 (width 128: of 256); of all key heads and sequences fewer than 2^24 (2^23),
 * else LOZA_ERR_SHAPE.
 */
int loza_ssa_extend_tree(const void *q, const void *k, const void *v, const int32_t *block_table, const int32_t *seqlens,
                         const int32_t *tree_lens, const int64_t *masks, void *out, float *lse, int B, int Hq, int Hkv,
                         int64_t S_max, int64_t num_pages, int page_size, int max_pages_per_seq, int n, int d_qk, int d_v,
                         int64_t sink_blocks, int64_t local_blocks, int64_t block, float scale, void *workspace,
                         size_t workspace_bytes, void *stream);
size_t loza_ssa_extend_tree_workspace_bytes(int B, int Hq, int Hkv, int64_t S_max, int n, int d_qk, int d_v,
                                            int64_t sink_blocks, int64_t local_blocks, int64_t block);

/* Host-only (ours), for tests and tools: the loza_kernel that a tree call of these sizes runs with scratch memory (scratch != 0) or without;
 * *n_splits (may be NULL): the workgroups that share the keys of a row. Negative on sizes that the call refuses. */
int loza_ssa_extend_tree_kernel(int B, int Hq, int Hkv, int64_t S_max, int n, int d_qk, int64_t sink_blocks, int64_t local_blocks,
                                int64_t block, int scratch, int *n_splits);

/*
 * Which drafts hold, and the token after them, from given random numbers, such that tokens are distributed as the target's
 * (recursive rejection sampling).
 *   target [B, n, V] fp32: probabilities after node r     draft [B, n, V] fp32: those that the children of node r were drawn from,
 *           independently; NULL: the drafts were not drawn at random
 *   tokens, parents [B, n] int32 (a node with a token outside [0, V) is skipped; tokens[b, 0] is not read), tree_lens [B] int32 (cut to [0, n])
 *   u_accept [B, n], u_next [B] fp32 in [0, 1)
 * From node 0 on: w = target, s = 1; the children x of the node are tried in order. Taken if u_accept q(x) s < w(x): on from there.
 * Else w = max(w - s q, 0), s = the sum of w. (Without draft q(x) = 1, w loses x, s the w(x).) Where no child is taken: the next token is
 * the first x whose w(0) + .. + w(x) exceeds u_next times the sum of all (w = target again if nothing is left of w).
 *   path [B, n] int32: nodes on the path, node 0 first, then -1     path_lens [B] int32: how many (0 for an empty tree)
 *   next_token [B] int32: the token after the path; -1 for an empty tree or a target row without weight
 *   workspace: loza_ssa_verify_tree_workspace_bytes, 16-byte aligned; contents ignored; two calls that overlap in time need two
 * A token whose target probability is negative or a NaN, or whose draft probability is a NaN, weighs 0. Infinite probabilities, and negative ones of the draft, are not allowed.
 * 1 <= n <= LOZA_TREE_MAX_NODES, B <= 65535, V <= 2^30. Sums and decisions in fp64, always in the same order.
 */
int loza_ssa_verify_tree(const float *target, const float *draft, const int32_t *tokens, const int32_t *parents, const int32_t *tree_lens,
                         const float *u_accept, const float *u_next, int32_t *path, int32_t *path_lens, int32_t *next_token,
                         int B, int n, int V, void *workspace, size_t workspace_bytes, void *stream);
size_t loza_ssa_verify_tree_workspace_bytes(int B, int n, int V);

/*
 * The rows of the accepted path to where a next step expects them: row slots[b, path[b, i]] becomes row slots[b, i] for all i < path_lens[b]
 * (the rows as they were before the call), in each of n_layers caches k_rows [n_layers, cache_rows, k_row_bytes], and v_rows likewise (NULL:
 * none). The request then has path_lens[b] rows more in its cache. Entries of path and slots outside their ranges are skipped; slots that the call
 * moves rows to or from must belong to one b. Row sizes: multiples of 16 bytes. B * n_layers <= 65535.
 */
int loza_ssa_keep_accepted(void *k_rows, void *v_rows, const int32_t *slots, const int32_t *path, const int32_t *path_lens, int B, int n,
                           int n_layers, int64_t cache_rows, int64_t k_row_bytes, int64_t v_row_bytes, void *stream);

/* Host-only (ours). Static string naming a status code. */
const char *loza_status_str(int status);

#ifdef __cplusplus
}
#endif
#endif /* LOZA_SSA_H */
