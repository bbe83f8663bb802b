// Pages of a cache beyond what a step needs (gfx950): shared with forks, copied, given back, moved to the front of the pool.
//
// A page belongs to the requests whose rows of the block table name it: one, and as many more as shared[page] says. Numbers of holders
// are changed by integer atomics, whose order does not show; lists are written in the order of requests or of page numbers, by counting
// what comes before. What bounds all of it but the copies: the latency of a few launches and of the loads in them that wait for each other (256 requests on 30,000
// pages: fork 2 + 5 us, give back 3 + 6 + 6; 40,000 pages renamed 5 + 6 + 9 + 7). The copies run at the memory's rate: 9,900 pages of 36 KB 147 us, 5.0 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_step.h"

namespace loza {

namespace {

template <typename T>
__device__ __forceinline__ T wave_total(T x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

__device__ __forceinline__ int64_t valid_count(const int32_t *count, int64_t num_free)
{
    const int64_t c = count[0];
    return c < 0 ? 0 : c < num_free ? c : num_free;
}

// Numbers before this thread's in a workgroup of 1,024 (each 0 .. 32: pages, or the bits of a word of them)
__device__ __forceinline__ int scan_before(int x, int32_t *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(sum, d, 64);
        if (lane >= d) sum += up;
    }
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    int before = sum - x;
    for (int i = 0; i < wave; ++i) before += lds[i];
    __syncthreads();
    return before;
}

// Small pools are done by one workgroup, with a number a page in LDS: one launch in the place of two (forks), three (pages given back) or four (compaction), which are also 3 us
// each of the host's time. us in a graph, several launches and one: 1,000 pages and 12 requests 5.4 and 4.0, 8.6 and 4.4, 13 and 4.0; 8,000 pages, 64 requests of 128 entries 5.7
// and 5.4, 10.3 and 8.6, 19 and 9; 256 requests of 64 6.0 and 7.1, 9.7 and 9.8, 19 and 11; 1,000 requests of 16 8 and 13, 10 and 16, 18 and 11.
constexpr int kSmallPages = 8192, kSmallRequests = 128, kSmallThreads = 1024;
constexpr int64_t kSmallRow = 512, kSmallTable = 32768;              // entries of a request; of all for a compaction
bool small(int64_t num_pages, int64_t B, int64_t max_pages) { return num_pages <= kSmallPages && B <= kSmallRequests && max_pages <= kSmallRow; }

// ---- forks ---------------------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void copy_ints_kernel(const int32_t *__restrict__ from, int32_t *__restrict__ to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from[i];
}

// What request b asks for: to become a copy of `source`, whose cache has `rows` rows
struct Fork {
    int source;
    int64_t rows;
    bool fits;
    int need;                      // pages: 1 for a page that is started and not full
};
__device__ __forceinline__ Fork fork_of(const ForkParams &p, int b)
{
    Fork f;
    f.source = p.from[b];
    f.fits = f.source >= 0 && f.source < p.B && p.cache_lens[b] == 0 && p.held[b] == 0;
    f.rows = f.fits ? p.cache_lens[f.source] : 0;
    const int held = f.fits ? p.held[f.source] : 0;
    if (f.rows < 0 || f.rows > (int64_t)p.max_pages << p.page_shift || held < 0 || held > p.max_pages) f.fits = false;
    f.need = f.fits && (f.rows & (((int64_t)1 << p.page_shift) - 1)) != 0;
    return f;
}

// Writes what becomes of request b; `before`: pages that the requests before it need
__device__ __forceinline__ void fork_made(const ForkParams &p, int b, const Fork &f, bool ok, int64_t full, int64_t first, int64_t before, int64_t count)
{
    const bool started = ok && f.need;
    int source = -1, target = -1;
    if (started) {
        source = p.block_table[(int64_t)f.source * p.max_pages + full];
        target = p.free_pages[count - 1 - before];
        p.block_table[(int64_t)b * p.max_pages + full] = target;
    }
    p.forked[b] = ok;
    p.cache_lens_after[b] = ok ? (int32_t)f.rows : p.cache_lens[b];
    p.held_after[b] = ok ? (int32_t)(full + f.need) : p.held[b];
    if (p.trimmed) p.trimmed_after[b] = ok ? (int32_t)first : p.trimmed[b];
    p.copy_from[b] = source;
    p.copy_to[b] = target;
    p.copy_rows[b] = started ? (int32_t)(f.rows & (((int64_t)1 << p.page_shift) - 1)) : 0;
}

// A workgroup a request. Pages are dealt out in the order of the requests: each adds up what those before its own need.
__global__ __launch_bounds__(256) void pages_fork_kernel(const ForkParams p)
{
    __shared__ int64_t s_sum[4];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int64_t count = valid_count(p.free_count, p.num_free);
    const Fork f = fork_of(p, b);                  // (asked for before there is anything to wait for)
    int64_t before = 0;
    const int upto = b == 0 ? p.B : b;             // (the first one adds up all, for what is left)
    for (int i = tid; i < upto; i += 256) before += fork_of(p, i).need;
    before = wave_total(before);
    if ((tid & 63) == 0) s_sum[tid >> 6] = before;
    __syncthreads();
    before = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
    if (b == 0) {
        if (tid == 0) p.free_left[0] = (int32_t)(count - (before < count ? before : count));
        before = 0;
    }
    const bool ok = f.fits && (f.need == 0 || before < count);
    const int64_t full = ok ? f.rows >> p.page_shift : 0;
    int64_t first = 0;                             // pages of the source from here on, and those of the sink, are still its own
    if (p.trimmed && ok) first = p.trimmed[f.source];
    int32_t *to = p.block_table + (int64_t)b * p.max_pages;
    const int32_t *from = p.block_table + (int64_t)(ok ? f.source : b) * p.max_pages;
    for (int64_t i = tid; i < full; i += 256) {
        const int page = from[i];
        to[i] = page;
        if ((i < p.sink_pages || i >= first) && page >= 0 && page < p.num_pages) atomicAdd(&p.shared_after[page], 1);
    }
    if (tid == 0) fork_made(p, b, f, ok, full, first, before, count);
}

__global__ __launch_bounds__(kSmallThreads) void pages_fork_small_kernel(const ForkParams p)
{
    __shared__ int32_t s_shared[kSmallPages], s_source[kSmallRequests], s_full[kSmallRequests], s_first[kSmallRequests], s_scan[16];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, pages = (int)p.num_pages;
    const int64_t count = valid_count(p.free_count, p.num_free);
    Fork f{-1, 0, false, 0};
    if (tid < p.B) f = fork_of(p, tid);
    for (int i = tid; i < pages; i += kSmallThreads) s_shared[i] = p.shared[i];
    const int before = scan_before(f.need, s_scan);
    const bool ok = f.fits && (f.need == 0 || before < count);
    const int full = ok ? (int)(f.rows >> p.page_shift) : 0, first = p.trimmed && ok ? p.trimmed[f.source] : 0;
    if (tid < p.B) {
        s_source[tid] = f.source;
        s_full[tid] = full;
        s_first[tid] = first;
        fork_made(p, tid, f, ok, full, first, before, count);
    }
    if (tid == kSmallThreads - 1) {
        const int64_t all = before + f.need;
        p.free_left[0] = (int32_t)(count - (all < count ? all : count));
    }
    __syncthreads();
    for (int b = wave; b < p.B; b += kSmallThreads / 64) {           // a wave a request
        const int32_t *from = p.block_table + (int64_t)s_source[b] * p.max_pages;
        int32_t *to = p.block_table + (int64_t)b * p.max_pages;
        for (int i = lane; i < s_full[b]; i += 64) {
            const int page = from[i];
            to[i] = page;
            if ((i < p.sink_pages || i >= s_first[b]) && page >= 0 && page < pages) atomicAdd(&s_shared[page], 1);
        }
    }
    __syncthreads();
    for (int i = tid; i < pages; i += kSmallThreads) p.shared_after[i] = s_shared[i];
}

// ---- copies ---------------------------------------------------------------------------------------------

// Workgroups take pieces of 16 KB of the pages of all layers in turn.
constexpr int kPiece = 256 * 16 * 4;

__global__ __launch_bounds__(256) void pages_copy_kernel(const CopyParams p)
{
    int64_t n = p.n;
    if (p.count) {
        const int64_t c = p.count[0];
        n = c < 0 ? 0 : c < n ? c : n;
    }
    const int64_t k_bytes = p.k_row * p.page_size, v_bytes = p.v_row * p.page_size;
    const int k_pieces = (int)((k_bytes + kPiece - 1) / kPiece), v_pieces = (int)((v_bytes + kPiece - 1) / kPiece), pieces = k_pieces + v_pieces;
    const int64_t items = n * p.layers * pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t il = item / pieces, i = il / p.layers, layer = il - i * p.layers;
        const int piece = (int)(item - il * pieces);
        const int64_t from = p.from[i], to = p.to[i];
        if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages || from == to) continue;
        int64_t rows = p.rows ? p.rows[i] : p.page_size;
        rows = rows < 0 ? 0 : rows < p.page_size ? rows : p.page_size;
        const bool values = piece >= k_pieces;
        const int64_t page_bytes = values ? v_bytes : k_bytes, bytes = rows * (values ? p.v_row : p.k_row);
        char *pages = (values ? p.v_pages : p.k_pages) + layer * p.num_pages * page_bytes;
        const int64_t at = (int64_t)(piece - (values ? k_pieces : 0)) * kPiece + threadIdx.x * 16;
        const char *x = pages + from * page_bytes;
        char *y = pages + to * page_bytes;
        u32x4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k * 4096 < bytes) v[k] = *(const u32x4 *)(x + at + k * 4096);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k * 4096 < bytes) *(u32x4 *)(y + at + k * 4096) = v[k];
    }
}

// ---- pages given back ----------------------------------------------------------------------------------
//
// left[page] starts as the number of holders beyond the first; each entry that is given up takes one off, and the one that finds 0 was
// the last and sets the page's bit. Freed pages go to the list by number: the workgroup of kPageGroup pages counts the bits before its own. (A number
// of freed pages for each group, added to by atomics, had the adds to one address wait for each other: 48 us for 10,000 pages.)

__global__ __launch_bounds__(256) void free_start_kernel(const FreeParams p)
{
    const int64_t words = (p.num_pages + 31) / 32;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.num_pages; i += (int64_t)gridDim.x * 256) p.left[i] = p.shared && p.shared[i] > 0 ? p.shared[i] : 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) p.freed[i] = 0;
}

// Entries [0, sink) and [first, upto) of request b's row are given up; `write`: and what the request has then is written
struct GivenUp {
    int64_t sink, first, upto;
};
__device__ __forceinline__ GivenUp given_up(const FreeParams &p, int b, bool write)
{
    const int64_t size = (int64_t)1 << p.page_shift, len = p.cache_lens[b], held = p.held[b];
    const int trimmed = p.trimmed ? p.trimmed[b] : 0;
    const bool fits = len >= 0 && len <= (int64_t)p.max_pages * size && held >= 0 && held <= p.max_pages;
    const bool ends = fits && p.ending && p.ending[b] != 0;
    const int64_t used = (len + size - 1) >> p.page_shift, have = held > used ? held : used;
    const int64_t first = trimmed > p.sink_pages ? trimmed : p.sink_pages;      // entries [0, sink_pages) and [first, have) are the request's
    int64_t upto = first;
    if (ends) {
        upto = have;
    } else if (fits && p.trimmed) {
        const int64_t seen = (int64_t)window_begin_of((int)len, p.window, p.block) >> p.page_shift;
        upto = seen > first ? seen : first;
    }
    if (write) {
        p.cache_lens_after[b] = ends ? 0 : (int32_t)len;
        p.held_after[b] = ends ? 0 : (int32_t)held;
        if (p.trimmed) p.trimmed_after[b] = ends ? 0 : upto > p.sink_pages ? (int32_t)(upto > trimmed ? upto : trimmed) : trimmed;
    }
    if (!fits) return GivenUp{0, 0, 0};
    return GivenUp{!ends ? 0 : p.sink_pages < have ? p.sink_pages : have, first, upto < have ? upto : have};
}

__global__ __launch_bounds__(256) void free_mark_kernel(const FreeParams p)
{
    const int b = blockIdx.x;
    const GivenUp g = given_up(p, b, blockIdx.y == 0 && threadIdx.x == 0);
    const int32_t *table = p.block_table + (int64_t)b * p.max_pages;
    const int64_t step = (int64_t)gridDim.y * 256, me = (int64_t)blockIdx.y * 256 + threadIdx.x;
    auto give = [&](int64_t i) {
        const int page = table[i];
        if (page < 0 || page >= p.num_pages) return;
        if (atomicSub(&p.left[page], 1) == 0) atomicOr(&p.freed[page >> 5], 1u << (page & 31));
    };
    for (int64_t i = me; i < g.sink; i += step) give(i);
    for (int64_t i = g.first + me; i < g.upto; i += step) give(i);
}

// How many of the bits below `limit` are set, by a workgroup of 1,024
__device__ __forceinline__ int64_t bits_below(const uint32_t *bits, int64_t limit, int64_t *lds)
{
    int64_t sum = 0;
    const int64_t words = limit / 32;
    for (int64_t i = threadIdx.x * 4; i + 4 <= words; i += 4096) {
        const u32x4 x = *(const u32x4 *)(bits + i);
        sum += __popc(x[0]) + __popc(x[1]) + __popc(x[2]) + __popc(x[3]);
    }
    if (threadIdx.x < 4) {                                           // up to three whole words, and a part of one
        const int64_t i = words / 4 * 4 + threadIdx.x;
        if (i * 32 < limit) {
            const uint32_t x = bits[i];
            sum += __popc(i < words ? x : x & ((1u << (limit & 31)) - 1));
        }
    }
    sum = wave_total(sum);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0;
    for (int i = 0; i < 16; ++i) sum += lds[i];
    __syncthreads();
    return sum;
}

// A workgroup a group of kPageGroup pages, 4 a thread
__global__ __launch_bounds__(1024) void free_append_kernel(const FreeParams p)
{
    __shared__ int64_t s_sum[16];
    __shared__ int32_t s_scan[16];
    const int64_t count = valid_count(p.free_count, p.num_free), page0 = (int64_t)blockIdx.x * kPageGroup + threadIdx.x * 4;
    int left[4], mine = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) left[k] = page0 + k < p.num_pages ? p.left[page0 + k] : 0;
    const int64_t before = bits_below(p.freed, (int64_t)blockIdx.x * kPageGroup, s_sum);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        mine += left[k] < 0;
        if (p.shared && page0 + k < p.num_pages) p.shared_after[page0 + k] = left[k] < 0 ? 0 : left[k];
    }
    int64_t at = count + before + scan_before(mine, s_scan);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (left[k] < 0) {
            if (at < p.num_free) p.free_pages[at] = (int32_t)(page0 + k);
            ++at;
        }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 1023) p.free_after[0] = (int32_t)(at < p.num_free ? at : p.num_free);   // (behind the last one's own)
}

__global__ __launch_bounds__(kSmallThreads) void pages_free_small_kernel(const FreeParams p)
{
    __shared__ int32_t s_left[kSmallPages], s_scan[16];
    __shared__ GivenUp s_given[kSmallRequests];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, pages = (int)p.num_pages;
    const int64_t count = valid_count(p.free_count, p.num_free);
    if (tid < p.B) s_given[tid] = given_up(p, tid, true);
    for (int i = tid; i < pages; i += kSmallThreads) s_left[i] = p.shared && p.shared[i] > 0 ? p.shared[i] : 0;
    __syncthreads();
    for (int b = wave; b < p.B; b += kSmallThreads / 64) {           // a wave a request
        const GivenUp g = s_given[b];
        const int32_t *table = p.block_table + (int64_t)b * p.max_pages;
        auto give = [&](int64_t i) {
            const int page = table[i];
            if (page >= 0 && page < pages) atomicSub(&s_left[page], 1);
        };
        for (int64_t i = lane; i < g.sink; i += 64) give(i);
        for (int64_t i = g.first + lane; i < g.upto; i += 64) give(i);
    }
    __syncthreads();
    // 8 pages a thread, in order
    constexpr int kEach = kSmallPages / kSmallThreads;
    int left[kEach], mine = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int page = tid * kEach + k;
        left[k] = page < pages ? s_left[page] : 0;
        mine += left[k] < 0;
        if (p.shared && page < pages) p.shared_after[page] = left[k] < 0 ? 0 : left[k];
    }
    int64_t at = count + scan_before(mine, s_scan);
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        if (left[k] < 0) {
            if (at < p.num_free) p.free_pages[at] = tid * kEach + k;
            ++at;
        }
    if (tid == kSmallThreads - 1) p.free_after[0] = (int32_t)(at < p.num_free ? at : p.num_free);
}

// ---- the pool tidied ------------------------------------------------------------------------------------
//
// With u pages in use, those from u on move to the free ones below u, each list by number: the i-th to the i-th.

__global__ __launch_bounds__(256) void compact_start_kernel(const CompactParams p)
{
    const int64_t words = (p.num_pages + 31) / 32;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) p.free_bits[i] = 0;
}

__global__ __launch_bounds__(256) void compact_mark_kernel(const CompactParams p)
{
    const int64_t count = valid_count(p.free_count, p.num_free);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int page = p.free_pages[i];
        if (page < 0 || page >= p.num_pages) continue;
        atomicOr(&p.free_bits[page >> 5], 1u << (page & 31));
    }
}

// A workgroup a group of pages: the lists of copies, each page's place in them, and the new free list
__global__ __launch_bounds__(1024) void compact_lists_kernel(const CompactParams p)
{
    __shared__ int64_t s_sum[16];
    __shared__ int32_t s_scan[16];
    const int64_t before = bits_below(p.free_bits, (int64_t)blockIdx.x * kPageGroup, s_sum), all = bits_below(p.free_bits, p.num_pages, s_sum);
    const int64_t used = p.num_pages - all, holes = bits_below(p.free_bits, used, s_sum);
    const int64_t page0 = (int64_t)blockIdx.x * kPageGroup + threadIdx.x * 4, most = p.num_pages / 2;
    const uint32_t bits = page0 < p.num_pages ? p.free_bits[page0 >> 5] >> (page0 & 31) & 15u : 0u;
    int64_t frees = before + scan_before(__popc(bits), s_scan);         // before page0 + k
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t page = page0 + k;
        if (page >= p.num_pages) break;
        const bool is_free = bits >> k & 1;
        if (is_free && page < used) {
            p.copy_to[frees] = (int32_t)page;
            p.place[page] = (int32_t)frees;
        } else if (!is_free && page >= used) {
            const int64_t i = page - frees - (used - holes);
            p.copy_from[i] = (int32_t)page;
            p.place[page] = (int32_t)i;
        }
        if (page >= holes && page < most) p.copy_from[page] = p.copy_to[page] = -1;
        frees += is_free;
    }
    for (int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x; i < p.num_free; i += (int64_t)gridDim.x * 1024)
        p.free_pages_after[i] = i < all ? (int32_t)(p.num_pages - 1 - i) : -1;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.free_after[0] = (int32_t)all;
        p.n_copies[0] = (int32_t)holes;
    }
}

__global__ __launch_bounds__(256) void compact_rename_kernel(const CompactParams p)
{
    const int64_t used = p.num_pages - p.free_after[0], entries = (int64_t)p.B * p.max_pages, step = (int64_t)gridDim.x * 256;
    auto is_free = [&](int64_t page) { return p.free_bits[page >> 5] >> (page & 31) & 1u; };
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += step) {
        const int page = p.block_table[i];
        p.table_after[i] = page >= used && page < p.num_pages && !is_free(page) ? p.copy_to[p.place[page]] : page;
    }
    if (p.shared == nullptr) return;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.num_pages; i += step)
        p.shared_after[i] = i >= used ? 0 : p.shared[is_free(i) ? p.copy_from[p.place[i]] : i];
}

__global__ __launch_bounds__(kSmallThreads) void pages_compact_small_kernel(const CompactParams p)
{
    constexpr int kWords = kSmallPages / 32;
    __shared__ uint32_t s_bits[kWords];                              // free pages
    __shared__ int32_t s_before[kWords], s_scan[16], s_all;          // how many of them are in the words before
    __shared__ uint16_t s_from[kSmallPages / 2], s_to[kSmallPages / 2];
    const int tid = threadIdx.x, pages = (int)p.num_pages;
    const int64_t count = valid_count(p.free_count, p.num_free);
    if (tid < kWords) s_bits[tid] = 0;
    __syncthreads();
    for (int64_t i = tid; i < count; i += kSmallThreads) {
        const int page = p.free_pages[i];
        if (page >= 0 && page < pages) atomicOr(&s_bits[page >> 5], 1u << (page & 31));
    }
    __syncthreads();
    const int mine = tid < kWords ? __popc(s_bits[tid]) : 0, sum = scan_before(mine, s_scan);
    if (tid < kWords) s_before[tid] = sum;
    if (tid == kWords - 1) s_all = sum + mine;
    __syncthreads();
    auto is_free = [&](int page) { return s_bits[page >> 5] >> (page & 31) & 1u; };
    auto frees = [&](int page) { return s_before[page >> 5] + __popc(s_bits[page >> 5] & ((1u << (page & 31)) - 1)); };     // of the pages below
    const int all = s_all, used = pages - all, holes = all > 0 ? frees(used) : 0, most = pages / 2;
    for (int page = tid; page < pages; page += kSmallThreads) {
        const bool is = is_free(page);
        if (is && page < used) {
            s_to[frees(page)] = (uint16_t)page;
            p.copy_to[frees(page)] = page;
        } else if (!is && page >= used) {
            const int i = page - frees(page) - (used - holes);
            s_from[i] = (uint16_t)page;
            p.copy_from[i] = page;
        }
        if (page >= holes && page < most) p.copy_from[page] = p.copy_to[page] = -1;
    }
    for (int64_t i = tid; i < p.num_free; i += kSmallThreads) p.free_pages_after[i] = i < all ? (int32_t)(pages - 1 - i) : -1;
    if (tid == 0) {
        p.free_after[0] = all;
        p.n_copies[0] = holes;
    }
    __syncthreads();
    const int entries = p.B * p.max_pages;
    for (int i = tid; i < entries; i += kSmallThreads) {
        const int page = p.block_table[i];
        p.table_after[i] = page >= used && page < pages && !is_free(page) ? s_to[page - frees(page) - (used - holes)] : page;
    }
    if (p.shared == nullptr) return;
    for (int i = tid; i < pages; i += kSmallThreads) p.shared_after[i] = i >= used ? 0 : p.shared[is_free(i) ? s_from[frees(i)] : i];
}

unsigned blocks_for(int64_t n, int threads, int64_t most)
{
    const int64_t b = (n + threads - 1) / threads;
    return (unsigned)(b < 1 ? 1 : b < most ? b : most);
}

}  // namespace

hipError_t launch_pages_fork(const ForkParams &p, hipStream_t stream)
{
    if (small(p.num_pages, p.B, p.max_pages)) {
        hipLaunchKernelGGL(pages_fork_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(copy_ints_kernel, dim3(blocks_for(p.num_pages, 256, 1024)), dim3(256), 0, stream, p.shared, p.shared_after, p.num_pages);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(pages_fork_kernel, dim3((unsigned)p.B), dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyParams &p, hipStream_t stream)
{
    const int64_t pieces = (p.k_row * p.page_size + kPiece - 1) / kPiece + (p.v_row * p.page_size + kPiece - 1) / kPiece;
    // (step by step: the product of all may pass 64 bits)
    int64_t items = p.n < 2048 ? p.n : 2048;
    items = items * p.layers < 2048 ? items * p.layers : 2048;
    items = items * pieces < 2048 ? items * pieces : 2048;
    hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)items), dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_pages_free(const FreeParams &p, hipStream_t stream)
{
    if (small(p.num_pages, p.B, p.max_pages)) {
        hipLaunchKernelGGL(pages_free_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(free_start_kernel, dim3(blocks_for(p.num_pages, 256, 1024)), dim3(256), 0, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(free_mark_kernel, dim3((unsigned)p.B, blocks_for(p.max_pages, 1024, 16)), dim3(256), 0, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(free_append_kernel, dim3((unsigned)((p.num_pages + kPageGroup - 1) / kPageGroup)), dim3(1024), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactParams &p, hipStream_t stream)
{
    if (p.num_pages <= kSmallPages && p.num_free <= kSmallTable && (int64_t)p.B * p.max_pages <= kSmallTable) {
        hipLaunchKernelGGL(pages_compact_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(compact_start_kernel, dim3(blocks_for(p.num_pages / 32 + 1, 256, 256)), dim3(256), 0, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(compact_mark_kernel, dim3(blocks_for(p.num_free, 256, 1024)), dim3(256), 0, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(compact_lists_kernel, dim3((unsigned)((p.num_pages + kPageGroup - 1) / kPageGroup)), dim3(1024), 0, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int64_t entries = (int64_t)p.B * p.max_pages;
    hipLaunchKernelGGL(compact_rename_kernel, dim3(blocks_for(entries > p.num_pages ? entries : p.num_pages, 1024, 2048)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace loza
