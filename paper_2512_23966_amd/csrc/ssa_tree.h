// A tree of drafted tokens as the queries of an extend: which keys a node sees.
//
// The nodes of sequence b are the last tree_lens[b] of its seqlens[b] cache rows, P rows come before them. Node r carries a mask: bit
// a says that it sees node a. Its position is P plus the nodes it sees, itself not counted; of the P rows it sees what the
// pattern gives that position, and of the nodes of its mask, the k-th of which sits at position P + k, those that are in the
// sink or in the window.
#ifndef LOZA_SSA_TREE_H
#define LOZA_SSA_TREE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_kernels.h"

namespace loza {

struct TreeSpan {
    int64_t L, P;        // valid cache rows, and those before the tree
    int nodes;
};
__device__ __forceinline__ TreeSpan tree_span(const FwdParams &p, int b)
{
    TreeSpan s;
    s.L = (int64_t)p.seqlens[b] < p.S ? (int64_t)p.seqlens[b] : p.S;
    if (s.L < 0) s.L = 0;
    int n = p.tree_lens[b];
    n = n < 0 ? 0 : n < p.q_len ? n : p.q_len;
    s.nodes = n < s.L ? n : (int)s.L;
    s.P = s.L - s.nodes;
    return s;
}

struct TreeRow {
    uint64_t mask;       // nodes that the row sees
    int w_lo;            // first key of its window
    bool seen;           // false: padding, or a node without a mask: it sees nothing
};
// In the place of the last key before the tree for a row that sees nothing. Its scores are masked where tiles are; where a tile takes no mask they
// are not, and its sums and its results are dropped at the end, by a select: 0 times what a value that is not finite left would be a NaN. Its query,
// which nobody need have written, is taken as 0: a NaN there had every tile's softmax done twice, an infinity moved the reference of the rows beside it.
constexpr int kNothing = -2;

__device__ __forceinline__ TreeRow tree_row(const FwdParams &p, const TreeSpan &s, int b, int r)
{
    TreeRow t;
    const uint64_t there = s.nodes < 64 ? ((uint64_t)1 << s.nodes) - 1 : ~(uint64_t)0;
    t.mask = r < s.nodes ? (uint64_t)p.tree_masks[(int64_t)b * p.q_len + r] & there : 0;
    t.seen = t.mask != 0;
    const int i = (int)s.P + __popcll(t.mask) - 1;
    t.w_lo = window_begin_of(i < 0 ? 0 : i, p.window, p.block);
    // nodes of the path whose positions are behind the window (few windows are shorter than a path) and not in the sink
    const int cut = t.w_lo - (int)s.P, sink = p.n_sink - (int)s.P;
    if (cut > 0) {
        uint64_t keep = 0, left = t.mask;
        for (int k = 0; left != 0; ++k, left &= left - 1)
            if (k >= cut || k < sink) keep |= left & -left;
        t.mask = keep;
    }
    return t;
}

// Partial results of tiles whose keys several workgroups share (trees): blocks of 32 rows x 128 columns as a wave's accumulators hold them, which it
// stores 1 KB an instruction (as rows of the result, an instruction touches 32 of them: 4 sequences of 8 nodes, wide shape, 68 -> 64 us).
// [row blocks of all (batch, key head)s][splits][column blocks][4 x 4][64 lanes][4], and of each row block and split 32 maxima, sums
// and rounded sums.
constexpr int kBlockFloats = 32 * 128;
__host__ __device__ __forceinline__ int tree_row_blocks(int64_t rows) { return (int)((rows + 31) / 32); }
__host__ __device__ __forceinline__ int64_t tree_part_floats(int64_t blocks, int n_splits, int d_v) { return blocks * n_splits * (d_v / 128) * kBlockFloats; }
// Row block `rb` (of its (batch, key head)) of split `split`: where its columns [128 cb, 128 cb + 128) are, and its maxima and sums
__device__ __forceinline__ float *tree_part_o(const FwdParams &p, int64_t bg, int rb, int split, int cb, int d_v)
{
    const int64_t block = bg * tree_row_blocks((int64_t)p.q_len * p.G) + rb;
    return p.part_o + ((block * p.n_splits + split) * (d_v / 128) + cb) * kBlockFloats;
}
__device__ __forceinline__ float *tree_part_ml(const FwdParams &p, int64_t bg, int rb, int split)
{
    return p.part_ml + ((bg * tree_row_blocks((int64_t)p.q_len * p.G) + rb) * p.n_splits + split) * 96;
}

// Bits of nodes first .. first + 31 of a mask, those outside [0, 64) clear. (first > -2^31 + 64)
__device__ __forceinline__ uint32_t tree_bits(uint64_t mask, int first)
{
    const uint64_t up = first < 64 ? mask >> (first & 63) : 0, down = first > -64 ? mask << (-first & 63) : 0;
    return (uint32_t)(first >= 0 ? up : down);
}

}  // namespace loza
#endif
