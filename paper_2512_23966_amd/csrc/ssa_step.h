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

struct KeepParams {
    char *k_rows, *v_rows;
    const int32_t *slots, *path, *path_lens;
    int B, n, layers;
    int64_t cache_rows, k_bytes, v_bytes;
};
hipError_t launch_keep_accepted(const KeepParams &p, hipStream_t stream);

}  // namespace loza
#endif
