// Internal interface of the kernels around a decode step (ssa_rope.hip, ssa_step.hip) with the C-ABI translation unit.
#ifndef LOZA_SSA_STEP_H
#define LOZA_SSA_STEP_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace loza {

// Nodes of a tree of drafted tokens: an ancestor set is one 64-bit word, a node a lane of a wave.
constexpr int kTreeNodes = 64;

struct TablesParams {
    const int32_t *cache_lens, *new_lens, *parents, *free_pages, *free_count;
    int32_t *block_table, *granted, *seqlens, *positions, *slots, *free_left;
    int64_t *masks;
    const int32_t *held;          // pages each request has (null: what its rows need), and what it has after the call
    int32_t *held_after;
    int B, n, page_shift, max_pages;
    int64_t num_free, num_pages;
};
hipError_t launch_step_tables(const TablesParams &p, hipStream_t stream);

// One tensor of heads that are rotated (strides in elements)
struct RopeHeads {
    const void *x;
    void *out;
    int64_t x_token, x_head, out_token, out_head;
    int H, d, rot_begin;
};
struct RopeParams {
    RopeHeads q, k;               // k.H == 0: a plain rotation of q alone; else k.out is the cache, row slots[t] of it
    const void *v;                // values that go to the cache as they are (may be null)
    void *v_rows;
    int64_t v_token, v_head;
    int d_v;
    const int32_t *positions, *slots;
    const double *freq;
    int64_t T, cache_rows;
    int rot;
    bool interleaved, inverse;
    float mscale;
};
// bytes of an element: 2 (bf16) or 4 (fp32)
hipError_t launch_rope(const RopeParams &p, int elem_bytes, hipStream_t stream);

// One tensor of heads that are normed over [norm_begin, norm_begin + norm_dim) (0: not) and rotated
struct NormHeads {
    RopeHeads r;
    const float *w;               // [norm_dim]; null: ones
    int norm_begin, norm_dim;
    int lanes;                    // of the group that takes a head (the launch's)
};
constexpr int kNormPartials = 768;    // partial sums of a weight's gradient, at most: workgroups, three of which fit a compute unit
struct NormParams {
    NormHeads q, k;               // k.r.H == 0: q alone; else k.r.out is the cache, row slots[t] of it
    const void *v;
    void *v_rows;
    int64_t v_token, v_head;
    int d_v;
    const int32_t *positions, *slots;
    const double *freq;
    int64_t T, cache_rows;
    int rot;
    bool interleaved;
    float mscale, eps;
    // the gradient (dout not null): q.r.x is the forward's input, q.r.out its gradient
    const void *dout;
    int64_t dout_token, dout_head;
    float *dw, *partial;          // null: not wanted; [kNormPartials, norm_dim]
};
hipError_t launch_norm_rope(const NormParams &p, int elem_bytes, hipStream_t stream);

struct VerifyParams {
    const float *target, *draft;
    const int32_t *tokens, *parents, *tree_lens;
    const float *u_accept, *u_next;
    int32_t *path, *path_lens, *next_token;
    double *partial;              // [B, rounds, slices] sums of the residual over slices of the vocabulary
    int B, n, V;
    int slices, slice_len, rounds;
    bool quads;                   // rows of target and draft are alike in their alignment to 16 bytes
};
// slices, slice_len and rounds of a call (host arithmetic on sizes), and the bytes of `partial`
void verify_plan(VerifyParams &p, bool draft);
hipError_t launch_verify_tree(const VerifyParams &p, hipStream_t stream);

constexpr int kMostBias = 1024;   // biased tokens of a request, at most
struct ProbsParams {
    const void *logits;           // [B, n] rows, logits_row elements apart
    int64_t logits_row;
    const int32_t *tokens;        // [B, n], with masks: the nodes of the trees
    const int64_t *masks;
    const int32_t *tree_lens;
    const uint16_t *seen;         // [B] rows, seen_row elements apart
    int64_t seen_row;
    const float *repetition, *frequency, *presence, *temperature;
    const int32_t *bias_tokens;
    const float *bias_values;
    int n_bias;
    const int32_t *allowed;       // [B, n, words]
    float *probs;
    float *stats;                 // [B n, slices] of 16 bytes: largest logit, sum, first token
    int B, n, V, words;
    int slices, slice_len;
};
// words, slices and slice_len of a call (host arithmetic on sizes)
void probs_plan(ProbsParams &p);
hipError_t launch_token_probs(const ProbsParams &p, int elem_bytes, hipStream_t stream);

struct CountParams {
    const int32_t *tokens, *path, *lens, *prompt_lens, *fresh;
    uint16_t *seen;
    int64_t seen_row;
    int B, n, V;
};
hipError_t launch_count_tokens(const CountParams &p, hipStream_t stream);

struct ForkParams {
    const int32_t *from, *cache_lens, *held, *trimmed, *free_pages, *free_count, *shared;
    int32_t *block_table, *forked, *cache_lens_after, *held_after, *trimmed_after, *copy_from, *copy_to, *copy_rows, *free_left, *shared_after;
    int B, page_shift, max_pages;
    int64_t num_free, num_pages, sink_pages;
};
hipError_t launch_pages_fork(const ForkParams &p, hipStream_t stream);

struct CopyParams {
    char *k_pages, *v_pages;
    const int32_t *from, *to, *rows, *count;
    int64_t n, num_pages, k_row, v_row;   // bytes of a row (v_row 0: no values)
    int layers, page_size;
};
hipError_t launch_pages_copy(const CopyParams &p, hipStream_t stream);

constexpr int kPageGroup = 4096;      // pages a workgroup counts
struct FreeParams {
    const int32_t *ending, *cache_lens, *held, *trimmed, *block_table, *shared, *free_count;
    int32_t *free_pages, *cache_lens_after, *held_after, *trimmed_after, *free_after, *shared_after;
    int32_t *left;                // workspace: [num_pages], and a bit a page
    uint32_t *freed;
    int B, page_shift, max_pages, window, block;
    int64_t num_free, num_pages, sink_pages;
};
hipError_t launch_pages_free(const FreeParams &p, hipStream_t stream);

struct CompactParams {
    const int32_t *block_table, *free_pages, *free_count, *shared;
    int32_t *table_after, *free_pages_after, *free_after, *shared_after, *copy_from, *copy_to, *n_copies;
    int32_t *place;               // workspace: [num_pages], and a bit a page
    uint32_t *free_bits;
    int B, max_pages;
    int64_t num_free, num_pages;
};
hipError_t launch_pages_compact(const CompactParams &p, hipStream_t stream);

struct KeepParams {
    char *k_rows, *v_rows;
    const int32_t *slots, *path, *path_lens;
    int B, n, layers;
    int64_t cache_rows, k_bytes, v_bytes;
};
hipError_t launch_keep_accepted(const KeepParams &p, hipStream_t stream);

}  // namespace loza
#endif
