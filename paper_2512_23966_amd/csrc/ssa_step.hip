// What a decode step does around its attention (gfx950): block tables, slots, positions and ancestor masks from request
// lengths; verification of a tree of drafted tokens; the accepted rows moved to their places in the cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_step.h"

namespace loza {

namespace {

template <typename T>
__device__ __forceinline__ T wave_sum(T x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

// Sum over this lane and those before it
template <typename T>
__device__ __forceinline__ T wave_scan(T x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T up = __shfl_up(x, d, 64);
        if (lane >= d) x += up;
    }
    return x;
}

// ---- tables ------------------------------------------------------------------------------------------

// What request b asks for: pages it holds already (rows that a step added and that were not kept leave it more than its cache needs),
// and new ones (0 where its numbers are not possible).
struct Request {
    int64_t cache, add, have, need;
    bool fits;
};
__device__ __forceinline__ Request request_of(const TablesParams &p, int b)
{
    Request r;
    r.cache = p.cache_lens[b];
    r.add = p.new_lens[b];
    const int64_t size = (int64_t)1 << p.page_shift;
    const int64_t held = p.held ? p.held[b] : 0;
    r.fits = r.cache >= 0 && r.add >= 0 && r.add <= p.n && r.cache + r.add <= (int64_t)p.max_pages * size && held >= 0 && held <= p.max_pages;
    const int64_t now = (r.cache + size - 1) >> p.page_shift, then = (r.cache + r.add + size - 1) >> p.page_shift;
    r.have = r.fits ? (now > held ? now : held) : 0;
    r.need = r.fits && then > r.have ? then - r.have : 0;
    return r;
}

// A workgroup takes kTokens tokens of one request. Pages are dealt out in the order of the requests, so each workgroup adds up what the
// requests before its own take (a scan across workgroups would cost a launch; 512 requests read 2 KB each, out of L2). Bound by the latency
// of four loads that wait for each other: 16 trees of 64 nodes 3.7 us, 512 requests of 200 tokens 6.1.
constexpr int kTokens = 1024;

__global__ __launch_bounds__(256) void step_tables_kernel(const TablesParams p)
{
    __shared__ int64_t s_sum[4];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t count0 = p.free_count[0], count = count0 < 0 ? 0 : count0 < p.num_free ? count0 : p.num_free;
    int64_t before = 0;
    for (int i = tid; i < b; i += 256) before += request_of(p, i).need;
    before = wave_sum(before);
    if (lane == 0) s_sum[wave] = before;
    __syncthreads();
    before = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
    const Request me = request_of(p, b);
    const bool ok = me.fits && (me.need == 0 || before + me.need <= count);
    const int granted = ok ? (int)me.add : 0;
    int32_t *table = p.block_table + (int64_t)b * p.max_pages;
    // new pages come from the end of the free list
    auto new_page = [&](int64_t i) { return p.free_pages[count - 1 - before - i]; };
    auto slot_of = [&](int64_t row) -> int32_t {
        const int64_t i = row >> p.page_shift;
        const int64_t page = i < me.have ? (int64_t)table[i] : (int64_t)new_page(i - me.have);
        if (page < 0 || page >= p.num_pages) return -1;
        return (int32_t)((page << p.page_shift) + (row & (((int64_t)1 << p.page_shift) - 1)));
    };
    if (blockIdx.y == 0) {
        if (ok)
            for (int64_t i = tid; i < me.need; i += 256) table[me.have + i] = new_page(i);
        if (tid == 0) {
            p.granted[b] = granted;
            p.seqlens[b] = (int32_t)(me.cache + granted);
            if (p.held) p.held_after[b] = me.fits ? (int32_t)(me.have + (ok ? me.need : 0)) : p.held[b];
        }
    }
    const int64_t at = (int64_t)b * p.n;
    if (p.parents != nullptr) {
        // a node a lane; ancestor sets by pointer jumping: after k steps a node knows its 2^k nearest ancestors
        if (wave == 0) {
            const int up0 = lane < granted ? p.parents[at + lane] : -1;
            int up = up0 >= 0 && up0 < lane ? up0 : -1;
            uint64_t mask = (uint64_t)1 << lane;
#pragma unroll
            for (int k = 0; k < 6; ++k) {
                const int from = up < 0 ? lane : up;
                const uint64_t m = __shfl((unsigned long long)mask, from, 64);
                const int u = __shfl(up, from, 64);
                if (up >= 0) {
                    mask |= m;
                    up = u;
                }
            }
            if (lane < p.n) {
                const bool there = lane < granted;
                p.masks[at + lane] = there ? (int64_t)mask : 0;
                p.positions[at + lane] = there ? (int32_t)(me.cache + __popcll(mask) - 1) : -1;
                p.slots[at + lane] = there ? slot_of(me.cache + lane) : -1;
            }
        }
    } else {
        const int64_t first = me.cache + granted - p.n;              // position of row 0
        const int end = (int)((int64_t)blockIdx.y * kTokens + kTokens < p.n ? (int64_t)blockIdx.y * kTokens + kTokens : p.n);
        for (int r = blockIdx.y * kTokens + tid; r < end; r += 256) {
            const bool there = r >= p.n - granted;
            p.positions[at + r] = there ? (int32_t)(first + r) : -1;
            p.slots[at + r] = there ? slot_of(first + r) : -1;
        }
    }
    if (b == 0 && blockIdx.y == 0 && wave == 3) {
        // What is left: the largest sum of needs that the free list covers is taken. (One wave, 64 requests at a time.)
        int64_t sum = 0, taken = 0;
        for (int i0 = 0; i0 < p.B; i0 += 64) {
            const int64_t incl = sum + wave_scan<int64_t>(i0 + lane < p.B ? request_of(p, i0 + lane).need : (int64_t)0);
            sum = __shfl(incl, 63, 64);
            const uint64_t covered = __ballot(incl <= count);      // (sums do not fall: the first lanes)
            if (covered) taken = __shfl(incl, 63 - __builtin_clzll(covered), 64);
            if (~covered) break;
        }
        if (lane == 0) p.free_left[0] = (int32_t)(count - taken);
    }
}

// ---- verification ------------------------------------------------------------------------------------
//
// Recursive rejection sampling over a tree. At node r with target probabilities p and draft probabilities q, the children x_1,
// x_2 .. are tried in order: with residual weights w = p and their sum s = 1 at first, a child is taken if u q(x) s < w(x); else
// w becomes max(w - s q, 0), and s the sum of that. Since max(max(a - b, 0) - c, 0) = max(a - b - c, 0), w is max(p - c q, 0)
// with ONE number c, the sum of the s so far: a rejection costs a sum over the vocabulary and no memory. Drafts that are not random
// (no q) have q = 1 at the child's own token: w is p without the rejected tokens, s comes from the p(x) alone. Where no child is
// taken (or there is none) the next token is drawn from w: the first whose running sum exceeds u_next times the sum of all.
//
// All decisions need p and q at the drafted tokens only, which every wave loads at once, a node a lane; sums over the vocabulary
// are what takes time (1 MB a sum at 131,072 tokens). Everything is in 64 bits: a decision next to a border must not hang on the
// order of a sum.

// A wave's walk through the tree, stopped where a sum is needed that is not known yet.
struct Walk {
    int parent, token;             // of this lane's node
    float p, q, u;                 // target and draft probability of its token at its parent; its random number
    int nodes;
    // state
    int cur, last;                 // node, and the last of its children tried
    double c, s;                   // multiple of q taken off p; sum of the residual (1 at first)
    uint64_t gone;                 // rejected children of cur (drafts that are not random)
    bool stale;                    // s does not belong to c yet
    uint64_t on_path;              // nodes on the path
};

__device__ __forceinline__ void walk_start(Walk &w, const VerifyParams &v, int b)
{
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)b * v.n + (lane < v.n ? lane : 0);
    const int nodes = v.tree_lens[b];
    w.parent = v.parents[at];
    w.token = v.tokens[at];
    w.u = v.u_accept[at];
    w.nodes = nodes < 0 ? 0 : nodes < v.n ? nodes : v.n;
    if (lane == 0 || lane >= w.nodes || w.parent < 0 || w.parent >= lane || w.token < 0 || w.token >= v.V) {
        w.parent = w.token = -1;                   // nobody's child
        w.p = w.q = 0.f;
    } else {
        const int64_t row = ((int64_t)b * v.n + w.parent) * v.V + w.token;
        w.p = v.target[row];
        w.q = v.draft ? v.draft[row] : 1.f;
    }
    w.cur = 0;
    w.last = 0;
    w.c = 0;
    w.s = 1;
    w.gone = 0;
    w.stale = false;
    w.on_path = w.nodes > 0 ? 1 : 0;
}

// Value of lane r (the same r in every lane)
__device__ __forceinline__ int lane_value(int x, int r) { return __builtin_amdgcn_readlane(x, r); }
__device__ __forceinline__ double lane_value(float x, int r)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), r));
}

// Goes on until a sum of the residual at w.cur is needed to go on (true) or no child is left to try (false).
template <bool DRAFT>
__device__ __forceinline__ bool walk_on(Walk &w)
{
    const int lane = threadIdx.x & 63;
    for (;;) {
        const uint64_t left = __ballot(w.parent == w.cur && lane > w.last);
        if (left == 0) return false;
        if (w.stale) return true;
        const int r = __builtin_ctzll(left);
        const double p = lane_value(w.p, r), q = lane_value(w.q, r), u = lane_value(w.u, r);
        double a;
        if (DRAFT) {
            a = p - w.c * q;
            a = a > 0 ? a : 0;
        } else {
            a = !(p > 0) || (__ballot(w.token == lane_value(w.token, r)) & w.gone) ? 0 : p;
        }
        w.last = r;
        if (u * q * w.s < a) {
            w.cur = r;
            w.on_path |= (uint64_t)1 << r;
            w.c = 0;
            w.s = 1;
            w.gone = 0;
        } else if (DRAFT) {
            w.c += w.s;
            w.stale = true;
        } else {
            w.s -= a;
            w.gone |= (uint64_t)1 << r;
        }
    }
}

// The residual weights at a node: what a token's weight is, given its probabilities; 0 where one of them is a NaN, or the target's is negative.
template <bool DRAFT>
struct Residual {
    const float *p, *q;
    double c;
    uint64_t gone;                 // rejected children whose tokens are among those asked for
    int token;                     // of this lane's node

    __device__ __forceinline__ Residual(const Walk &w, const VerifyParams &v, int b, int x0, int x1)
    {
        const int64_t row = ((int64_t)b * v.n + w.cur) * v.V;
        p = v.target + row;
        q = DRAFT ? v.draft + row : nullptr;
        c = w.c;
        token = w.token;
        gone = DRAFT ? 0 : w.gone & __ballot(token >= x0 && token < x1);
    }
    __device__ __forceinline__ double weight(int x, float px, float qx) const
    {
        if constexpr (DRAFT) {
            const double a = (double)px - c * (double)qx;
            return a > 0 ? a : 0;
        } else {
            for (uint64_t g = gone; g; g &= g - 1) px = x == lane_value(token, __builtin_ctzll(g)) ? 0.f : px;
            return __builtin_amdgcn_fmed3f(px, 0.f, __builtin_inff());   // (of a NaN: the least of the others)
        }
    }
    __device__ __forceinline__ double at(int x) const { return weight(x, p[x], DRAFT ? q[x] : 0.f); }
};

// This wave's share of the sum over the slice [x0, x1), in every lane: thread `first` of `step` takes 4 tokens at a time, in 16-byte loads
// from the first address of that alignment on (quads: both rows have the same), and one of the up to 3 tokens before and behind those.
template <bool DRAFT>
__device__ __forceinline__ double wave_residual(const Residual<DRAFT> &r, bool quads, int x0, int x1, int first, int step)
{
    double sum = 0;
    if (quads) {
        int head = -(int)((uintptr_t)(r.p + x0) >> 2) & 3;
        head = head < x1 - x0 ? head : x1 - x0;
        const int tail = (x1 - x0 - head) & 3;
        if (first < head) sum += r.at(x0 + first);
        if (first < tail) sum += r.at(x1 - tail + first);
#pragma unroll 4
        for (int x = x0 + head + 4 * first; x < x1 - tail; x += 4 * step) {
            const float4 p = *(const float4 *)(r.p + x);
            float4 q = {0.f, 0.f, 0.f, 0.f};
            if constexpr (DRAFT) q = *(const float4 *)(r.q + x);
            sum += (r.weight(x, p.x, q.x) + r.weight(x + 1, p.y, q.y)) + (r.weight(x + 2, p.z, q.z) + r.weight(x + 3, p.w, q.w));
        }
    } else {
#pragma unroll 4
        for (int x = x0 + first; x < x1; x += step) sum += r.at(x);
    }
    return wave_sum(sum);
}

// The sum over all slices, always in the same order
__device__ __forceinline__ double slices_sum(const double *part, int n)
{
    double sum = 0;
    for (int i = threadIdx.x & 63; i < n; i += 64) sum += part[i];
    return wave_sum(sum);
}

// Round `round` of the sums over the vocabulary that a walk needs one after the other: each workgroup repeats the walk up to
// there (from the sums of the rounds before) and adds up its slice.
template <bool DRAFT>
__global__ __launch_bounds__(256) void verify_sum_kernel(const VerifyParams v, const int round)
{
    __shared__ double s_sum[4];
    const int b = blockIdx.y, slice = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double *part = v.partial + (int64_t)b * v.rounds * v.slices;
    Walk w;
    walk_start(w, v, b);
    if (w.nodes == 0) return;
    for (int k = 0; k < round; ++k) {
        if (!walk_on<DRAFT>(w)) return;                    // that round's sum was the last one
        w.s = slices_sum(part + k * v.slices, v.slices);
        w.stale = false;
    }
    walk_on<DRAFT>(w);
    const int x0 = slice * v.slice_len, x1 = x0 + v.slice_len < v.V ? x0 + v.slice_len : v.V;
    const double sum = wave_residual<DRAFT>(Residual<DRAFT>(w, v, b, x0, x1), v.quads, x0, x1, threadIdx.x, 256);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) part[round * v.slices + slice] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

constexpr int kMaxSlices = 256;

// The end of the walk (sums beyond those rounds are taken here, by one workgroup) and the next token.
template <bool DRAFT>
__global__ __launch_bounds__(1024) void verify_tree_kernel(const VerifyParams v)
{
    __shared__ double s_part[kMaxSlices], s_wave[16];
    __shared__ int s_first;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const double *part = v.partial + (int64_t)b * v.rounds * v.slices;
    const double u_next = v.u_next[b];             // (asked for before there is anything to wait for)
    Walk w;
    walk_start(w, v, b);
    if (w.nodes > 0) {
        auto sum_here = [&]() {
            __syncthreads();
            for (int s = wave; s < v.slices; s += 16) {
                const int x0 = s * v.slice_len, x1 = x0 + v.slice_len < v.V ? x0 + v.slice_len : v.V;
                const double sum = wave_residual<DRAFT>(Residual<DRAFT>(w, v, b, x0, x1), v.quads, x0, x1, lane, 64);
                if (lane == 0) s_part[s] = sum;
            }
            __syncthreads();
        };
        int k = 0;
        bool more;
        do {
            more = walk_on<DRAFT>(w);
            if (k < v.rounds) {
                __syncthreads();
                if (tid < v.slices) s_part[tid] = part[k * v.slices + tid];
                __syncthreads();
            } else {
                sum_here();
            }
            w.s = slices_sum(s_part, v.slices);
            w.stale = false;
            ++k;
        } while (more);
        if (!(w.s > 0)) {                                  // nothing is left of the residual (rounding): the target itself
            w.c = 0;
            w.gone = 0;
            sum_here();
            w.s = slices_sum(s_part, v.slices);
        }
        if (w.s > 0) {
            // the slice in which the running sum passes the threshold, then the token (every thread takes a run of tokens)
            double thr = u_next * w.s;
            double four[4], upto = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                four[i] = 4 * lane + i < v.slices ? s_part[4 * lane + i] : 0;
                upto += four[i];
            }
            upto = wave_scan(upto);
            const uint64_t beyond = __ballot(upto > thr);
            const int l = beyond ? __builtin_ctzll(beyond) : (v.slices - 1) / 4;
            double at = l > 0 ? __shfl(upto, l > 0 ? l - 1 : 0, 64) : 0;
            int slice = 4 * l;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const double part_i = __shfl(four[i], l, 64);
                if (slice == 4 * l + i && slice < v.slices - 1 && !(at + part_i > thr)) {
                    at += part_i;
                    ++slice;
                }
            }
            thr -= at;
            const int x0 = slice * v.slice_len, x1 = x0 + v.slice_len < v.V ? x0 + v.slice_len : v.V;
            const int per = (v.slice_len + 1023) / 1024;
            const Residual<DRAFT> res(w, v, b, 0, v.V);
            int a = x0 + tid * per, e = a + per < x1 ? a + per : x1;
            double mine = 0;
            for (int x = a; x < e; ++x) mine += res.at(x);
            const double incl = wave_scan(mine);
            if (lane == 63) s_wave[wave] = incl;
            if (tid == 0) s_first = 1023;
            __syncthreads();
            double base = 0;
            for (int i = 0; i < wave; ++i) base += s_wave[i];
            const uint64_t past = __ballot(base + incl > thr);
            if (lane == 0 && past) atomicMin(&s_first, wave * 64 + __builtin_ctzll(past));
            __syncthreads();
            // (the sums were added in another order than this loop adds: where the threshold is not passed after all, the last token
            // with a weight is taken, of this run or the nearest beside it)
            if (tid == s_first) {
                double run = base + (incl - mine);
                int pick = -1;
                if (per == 1 && mine > 0) pick = a;
                for (int x = pick < 0 ? a : e; x < e; ++x) {
                    const double wx = res.at(x);
                    if (!(wx > 0)) continue;
                    pick = x;
                    run += wx;
                    if (run > thr) break;
                }
                const int end = a < x1 ? e : x1;
                for (int x = end; x < v.V && pick < 0; ++x)
                    if (res.at(x) > 0) pick = x;
                for (int x = end - 1; x >= 0 && pick < 0; --x)
                    if (res.at(x) > 0) pick = x;
                v.next_token[b] = pick;
            }
        }
    }
    if (tid == 0 && !(w.nodes > 0 && w.s > 0)) v.next_token[b] = -1;
    if (wave == 0) {
        const int len = __popcll(w.on_path);
        if (lane == 0) v.path_lens[b] = len;
        if (lane >= len && lane < v.n) v.path[(int64_t)b * v.n + lane] = -1;
        if ((w.on_path >> lane) & 1) v.path[(int64_t)b * v.n + __popcll(w.on_path & (((uint64_t)1 << lane) - 1))] = lane;
    }
}

// ---- accepted rows -------------------------------------------------------------------------------------
//
// Row slots[path[i]] of the cache becomes row slots[i], for the nodes i < path_lens of the accepted path. A row may be both: the
// workgroup reads its columns of all rows before it writes any. Bound by latency (a path is a few rows of 1 KB, a layer).
constexpr int kKeepChunks = 16;    // 16-byte chunks of a row a workgroup takes: 64 rows of them are 4 a thread

__global__ __launch_bounds__(256) void keep_accepted_kernel(const KeepParams p)
{
    const int64_t b = blockIdx.y % p.B, layer = blockIdx.y / p.B;
    const int kc = (int)(p.k_bytes / 16), k_groups = (kc + kKeepChunks - 1) / kKeepChunks;
    const bool values = (int)blockIdx.x >= k_groups;
    const int64_t bytes = values ? p.v_bytes : p.k_bytes;
    const int c = ((int)blockIdx.x - (values ? k_groups : 0)) * kKeepChunks + (threadIdx.x & 15);
    char *rows = (values ? p.v_rows : p.k_rows) + layer * p.cache_rows * bytes;
    int len = p.path_lens[b];
    len = len < 0 ? 0 : len < p.n ? len : p.n;
    u32x4 x[4];
    int64_t to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int node = i * 16 + (threadIdx.x >> 4);
        to[i] = -1;
        if (node >= len || c * 16 >= bytes) continue;
        const int from = p.path[b * p.n + node];
        if (from < 0 || from >= p.n || from == node) continue;
        const int64_t src = p.slots[b * p.n + from], dst = p.slots[b * p.n + node];
        if (src < 0 || src >= p.cache_rows || dst < 0 || dst >= p.cache_rows) continue;
        x[i] = *(const u32x4 *)(rows + src * bytes + c * 16);
        to[i] = dst;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));      // the rows are here before any is overwritten
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (to[i] >= 0) *(u32x4 *)(rows + to[i] * bytes + c * 16) = x[i];
}

}  // namespace

hipError_t launch_step_tables(const TablesParams &p, hipStream_t stream)
{
    const int chunks = p.parents ? 1 : (p.n + kTokens - 1) / kTokens;
    hipLaunchKernelGGL(step_tables_kernel, dim3((unsigned)p.B, (unsigned)chunks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

// Slices: enough workgroups to fill the chip for a few sequences, at least 1,024 tokens each. Rounds of sums by all of them, a launch each of
// 2.5 us where there is nothing to add up, against some 10 for a sum over 131,072 tokens by one workgroup: none for up to 65,536 probabilities a
// sum of calls whose probabilities are still in a cache when they are small enough for one (32,000 tokens, one chain of 5 nodes: 9.1 us, with a round 10.7;
// from memory 16.7 and 14.6). A chain or drafts that are not random need one sum (131,072 tokens from memory, 16 sequences of 5 nodes: no round 36.8 us,
// one 20.0, two 23.2); wider trees of random drafts need as many as children are rejected (16 of 16 nodes: one round 44 us, three 33,
// four 37; one of 64: one 31, three 23, five 30; 16 of 64: one 99, three 81, five 65, six 61, eight 73). Measured on up to 16 trees; from some 64
// on slices are few (16 of 64 trees, 2 of 512), and a sum beyond the rounds, taken by one wave a slice, leaves most of its workgroup idle.
void verify_plan(VerifyParams &p, bool draft)
{
    int64_t slices = (1024 + p.B - 1) / p.B;
    if (slices > kMaxSlices) slices = kMaxSlices;
    if (slices > ((int64_t)p.V + 1023) / 1024) slices = ((int64_t)p.V + 1023) / 1024;
    p.slice_len = (int)(((p.V + slices - 1) / slices + 63) / 64 * 64);
    p.slices = (p.V + p.slice_len - 1) / p.slice_len;
    const int64_t sum = (int64_t)p.V * (draft ? 2 : 1);
    const bool cached = sum * p.B * p.n * 4 <= 64 << 20;
    p.rounds = sum <= 65536 && cached ? 0 : !draft || p.n <= 8 ? 1 : p.n <= 24 || p.B < 8 ? 3 : 5;
    p.quads = !draft || ((reinterpret_cast<uintptr_t>(p.target) ^ reinterpret_cast<uintptr_t>(p.draft)) & 15u) == 0;
}

template <bool DRAFT>
static hipError_t launch_verify_t(const VerifyParams &p, hipStream_t stream)
{
    for (int round = 0; round < p.rounds; ++round) {
        hipLaunchKernelGGL((verify_sum_kernel<DRAFT>), dim3((unsigned)p.slices, (unsigned)p.B), dim3(256), 0, stream, p, round);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((verify_tree_kernel<DRAFT>), dim3((unsigned)p.B), dim3(1024), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_verify_tree(const VerifyParams &p, hipStream_t stream)
{
    return p.draft ? launch_verify_t<true>(p, stream) : launch_verify_t<false>(p, stream);
}

hipError_t launch_keep_accepted(const KeepParams &p, hipStream_t stream)
{
    const int64_t groups = (p.k_bytes / 16 + kKeepChunks - 1) / kKeepChunks + (p.v_rows ? (p.v_bytes / 16 + kKeepChunks - 1) / kKeepChunks : 0);
    hipLaunchKernelGGL(keep_accepted_kernel, dim3((unsigned)groups, (unsigned)(p.B * p.layers)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace loza
