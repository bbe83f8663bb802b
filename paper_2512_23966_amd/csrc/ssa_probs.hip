// Probabilities of the next token from logits, under penalties for repeated tokens, biases and grammar masks (gfx950), and the
// record of a request's tokens that the penalties read.
//
// Token x of a row has the logit l, the number c of times it was said and whether it occurred at all (said, or in the prompt):
//     l' = l / repetition if l > 0, l * repetition otherwise, where it occurred;  l'' = l' - frequency c - presence (c > 0) + bias
// and no weight where the grammar does not allow it (or l'' is a NaN); p = exp((l'' - max) / T) / sum, or 1 at the first of the largest.
//
// What bounds it: memory, 4 bytes a token out and 2 or 4 in; so all of it is done on the way. The tokens of a tree's own nodes and the
// biased ones are a few hundred of 100,000: the pass over the row leaves them out (a bit each in LDS), and a thread each does them
// apart, so that the pass looks nothing up.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_rope.h"
#include "ssa_step.h"

namespace loza {

namespace {

constexpr int kUnit = 8;                         // tokens a thread takes at a time: 16 bytes of bf16 logits and of the record
constexpr int kThreads = 256, kStep = kUnit * kThreads;
constexpr int kMostSlice = 131072;               // tokens of a slice (a bit each in LDS)
constexpr int kMostSpecial = kTreeNodes + kMostBias;

// What a row's logits are changed by
struct Change {
    float rep, fre, pre;
    // Each operation rounded by itself, as a plain program does them: a token next to another must not win by a rounding left out.
    __device__ __forceinline__ float operator()(float l, bool occurred, int said) const
    {
#pragma clang fp contract(off)
        if (occurred) l = l > 0.f ? l / rep : l * rep;
        if (said > 0) {
            const float f = fre * (float)said;
            l = l - f;
            l = l - pre;
        }
        return l;
    }
};

// exp(d / T) for d <= 0: 2^(d c), c = log2(e) / T in two parts, the rounding of the product given back to first order
struct Weight {
    float hi, lo;
    __device__ __forceinline__ explicit Weight(float t)
    {
        const double c = 1.4426950408889634074 / (double)t;
        hi = (float)c;
        lo = (float)(c - (double)hi);
    }
    __device__ __forceinline__ float operator()(float d) const
    {
        const float h = d * hi, rest = __builtin_fmaf(d, lo, __builtin_fmaf(d, hi, -h)), p = __builtin_amdgcn_exp2f(h);
        return h < -150.f ? 0.f : __builtin_fmaf(p * rest, 0.693147180559945f, p);      // (-inf is such an h, too)
    }
};

// Largest logit, its first token, and the sum of the weights relative to it
struct Stat {
    float m, s;
    int32_t x, unused;
};
__device__ __forceinline__ float difference(float l, float m) { return l == m ? 0.f : l - m; }   // (of two infinities: 0)
__device__ __forceinline__ void merge(Stat &a, float m, float s, int32_t x, const Weight &w)
{
    if (m == LOZA_NEG_INF) return;
    if (m > a.m) {
        a.s = s + (a.m == LOZA_NEG_INF ? 0.f : a.s * w(difference(a.m, m)));
        a.m = m;
        a.x = x;
    } else {
        a.s += s * w(difference(m, a.m));
        if (m == a.m && x < a.x) a.x = x;
    }
}

template <typename E>
__device__ __forceinline__ void load_unit(const E *at, float (&l)[kUnit])
{
    u32x4 raw[sizeof(E) / 2];
    __builtin_memcpy(raw, at, sizeof(raw));      // (rows of odd vocabularies are aligned to their elements only)
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = __builtin_bit_cast(float, i & 1 ? raw[0][i / 2] & 0xffff0000u : raw[0][i / 2] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i) {
            const uint32_t x = raw[i / 4][i % 4];       // (a bit cast of a vector's element itself takes its first one)
            l[i] = __builtin_bit_cast(float, x);
        }
    }
}

// One row's slice [x0, x1): the tokens that are done apart, and what the pass over the others needs.
template <typename E>
struct Slice {
    const ProbsParams &p;
    const E *row;
    const uint16_t *seen;
    const uint8_t *allowed;
    int b, r, x0, x1, entries;
    Change change;
    int32_t *tok;                 // LDS: [entries] tokens done apart, -1 where they are not in the slice
    uint32_t *bits;               // LDS: a bit a token of the slice

    __device__ __forceinline__ Slice(const ProbsParams &p_, int64_t row_index, int slice, int32_t *tok_, uint32_t *bits_) : p(p_), tok(tok_), bits(bits_)
    {
        b = (int)(row_index / p.n);
        r = (int)(row_index - (int64_t)b * p.n);
        row = (const E *)p.logits + row_index * p.logits_row;
        seen = p.seen ? p.seen + (int64_t)b * p.seen_row : nullptr;
        allowed = p.allowed ? (const uint8_t *)(p.allowed + row_index * p.words) : nullptr;
        x0 = slice * p.slice_len;
        x1 = x0 + p.slice_len < p.V ? x0 + p.slice_len : p.V;
        change.rep = p.repetition ? p.repetition[b] : 1.f;
        change.fre = p.frequency ? p.frequency[b] : 0.f;
        change.pre = p.presence ? p.presence[b] : 0.f;
        const int nodes = p.masks ? p.n : 0;
        entries = nodes + p.n_bias;
        if (entries == 0) return;
        for (int i = threadIdx.x; i < (x1 - x0 + 31) / 32; i += kThreads) bits[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < entries; i += kThreads) {
            int x = -1;
            if (i < nodes) {
                const uint64_t path = (uint64_t)p.masks[row_index];
                if ((path >> i & 1) && i < length()) x = p.tokens[(int64_t)b * p.n + i];
            } else {
                x = p.bias_tokens[(int64_t)b * p.n_bias + i - nodes];
            }
            if (x < x0 || x >= x1) x = -1;
            tok[i] = x;
            if (x >= 0) atomicOr(&bits[(x - x0) >> 5], 1u << ((x - x0) & 31));
        }
        __syncthreads();
    }
    __device__ __forceinline__ int length() const
    {
        const int len = p.tree_lens ? p.tree_lens[b] : p.n;
        return len < p.n ? len : p.n;
    }
    // The changed logits of the tokens [x, x + 8); -inf for those done apart (whose bits come back), not allowed, or not there
    __device__ __forceinline__ uint32_t unit(int x, float (&l)[kUnit]) const
    {
        const uint32_t apart = entries ? ((const uint8_t *)bits)[(x - x0) >> 3] : 0u;
        uint32_t ok = allowed ? allowed[x >> 3] : 0xffu;
        if (x + kUnit <= p.V) {
            load_unit(row + x, l);
        } else {
            ok &= (1u << (p.V - x)) - 1;
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] = x + i < p.V ? Elem<E>::get(row[x + i]) : 0.f;
        }
        if (seen) {
            const Pack<uint16_t, kUnit> z = *(const Pack<uint16_t, kUnit> *)(seen + x);
            const u32x4 any = __builtin_bit_cast(u32x4, z);
            if (any[0] | any[1] | any[2] | any[3]) {
#pragma unroll
                for (int i = 0; i < kUnit; ++i) l[i] = change(l[i], z.e[i] != 0, z.e[i] & 0x7fff);
            }
        }
        ok &= ~apart;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = (ok >> i & 1) && l[i] == l[i] ? l[i] : LOZA_NEG_INF;
        return apart;
    }
    // The changed logit of entry i, and whether it is the one that stands for its token (the first of them)
    __device__ __forceinline__ bool special(int i, float &l) const
    {
#pragma clang fp contract(off)
        const int x = tok[i];
        if (x < 0) return false;
        for (int k = 0; k < i; ++k)
            if (tok[k] == x) return false;
        const int nodes = p.masks ? p.n : 0;
        const int z = seen ? seen[x] : 0;
        int said = z & 0x7fff;
        float bias = 0.f;
        for (int k = i; k < entries; ++k)
            if (tok[k] == x) {
                if (k < nodes) ++said;
                else bias = bias + p.bias_values[(int64_t)b * p.n_bias + k - nodes];
            }
        l = change(Elem<E>::get(row[x]), z >= 0x8000 || said > 0, said);
        l = l + bias;
        if (!(l == l) || (allowed && !(allowed[x >> 3] >> (x & 7) & 1))) l = LOZA_NEG_INF;
        return true;
    }
};

// Requests whose temperature is 0 (or otherwise none to divide by) take the largest logit.
__device__ __forceinline__ float temperature_of(const ProbsParams &p, int b)
{
    const float t = p.temperature ? p.temperature[b] : 1.f;
    return t >= 0x1p-126f && t <= 0x1p126f ? t : 0.f;
}

// Stat of a whole workgroup, in thread 0
__device__ __forceinline__ Stat workgroup_stat(Stat a, const Weight &w, Stat *lds)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const float m = __shfl_xor(a.m, d, 64), s = __shfl_xor(a.s, d, 64);
        const int x = __shfl_xor(a.x, d, 64);
        // (both lanes of a pair take the sum in the same order)
        Stat lo = a;
        const bool low = (threadIdx.x & d) == 0;
        float m2 = m, s2 = s;
        int x2 = x;
        if (!low) {
            lo.m = m; lo.s = s; lo.x = x;
            m2 = a.m; s2 = a.s; x2 = a.x;
        }
        merge(lo, m2, s2, x2, w);
        a = lo;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < kThreads / 64; ++i) merge(a, lds[i].m, lds[i].s, lds[i].x, w);
    return a;
}

constexpr Stat kNoStat = {LOZA_NEG_INF, 0.f, 0x7fffffff, 0};

template <typename E>
__global__ __launch_bounds__(kThreads) void token_stats_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ int32_t s_tok[kMostSpecial];
    __shared__ Stat s_stat[kThreads / 64];
    const int64_t row = blockIdx.x / p.slices;
    const int slice = (int)(blockIdx.x - row * p.slices);
    if (p.tree_lens && (int)(row % p.n) >= p.tree_lens[row / p.n]) return;
    const Slice<E> s(p, row, slice, s_tok, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    Stat a = kNoStat;
    for (int x = s.x0 + (int)threadIdx.x * kUnit; x < s.x1; x += kStep) {
        float l[kUnit];
        s.unit(x, l);
        float m = l[0];
#pragma unroll
        for (int i = 1; i < kUnit; ++i) m = fmaxf(m, l[i]);
        if (m > a.m) {
            if (t > 0.f) a.s = a.m == LOZA_NEG_INF ? 0.f : a.s * w(difference(a.m, m));
            a.m = m;
            int at = 0;
#pragma unroll
            for (int i = kUnit - 1; i >= 0; --i) at = l[i] == m ? i : at;
            a.x = x + at;
        }
        if (t > 0.f && a.m != LOZA_NEG_INF) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) a.s += w(difference(l[i], a.m));
        }
    }
    for (int i = threadIdx.x; i < s.entries; i += kThreads) {
        float l;
        if (s.special(i, l)) merge(a, l, 1.f, s.tok[i], w);
    }
    a = workgroup_stat(a, w, s_stat);
    if (threadIdx.x == 0) p.stats[(int64_t)blockIdx.x * 4] = a.m, p.stats[(int64_t)blockIdx.x * 4 + 1] = a.s, ((int32_t *)p.stats)[(int64_t)blockIdx.x * 4 + 2] = a.x;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void token_probs_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ int32_t s_tok[kMostSpecial];
    __shared__ Stat s_stat[kThreads / 64];
    const int64_t row = blockIdx.x / p.slices;
    const int slice = (int)(blockIdx.x - row * p.slices);
    if (p.tree_lens && (int)(row % p.n) >= p.tree_lens[row / p.n]) return;
    const Slice<E> s(p, row, slice, s_tok, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    Stat a = kNoStat;
    for (int i = threadIdx.x; i < p.slices; i += kThreads) {
        const float *at = p.stats + (row * p.slices + i) * 4;
        merge(a, at[0], at[1], ((const int32_t *)at)[2], w);
    }
    a = workgroup_stat(a, w, s_stat);
    __syncthreads();
    if (threadIdx.x == 0) s_stat[0] = a;
    __syncthreads();
    a = s_stat[0];
    const float inv = a.m == LOZA_NEG_INF ? 0.f : 1.f / a.s;
    const bool greedy = !(t > 0.f);
    auto prob = [&](float l, int x) { return greedy ? (x == a.x ? 1.f : 0.f) : l == LOZA_NEG_INF ? 0.f : w(difference(l, a.m)) * inv; };
    float *out = p.probs + row * p.V;
    for (int x = s.x0 + (int)threadIdx.x * kUnit; x < s.x1; x += kStep) {
        float l[kUnit];
        const uint32_t apart = s.unit(x, l);
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = prob(l[i], x + i);
        if (apart == 0 && x + kUnit <= p.V) {
            __builtin_memcpy(out + x, l, sizeof(l));
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i)
                if (!(apart >> i & 1) && x + i < p.V) out[x + i] = l[i];
        }
    }
    for (int i = threadIdx.x; i < s.entries; i += kThreads) {
        float l;
        if (s.special(i, l)) out[s.tok[i]] = prob(l, s.tok[i]);
    }
}

// ---- the record of a request's tokens -----------------------------------------------------------------------
//
// 16 bits a token of the vocabulary: bit 15, it occurs in the prompt; the others, how often it was said, which stops at 32,767.

__global__ __launch_bounds__(256) void clear_seen_kernel(const CountParams p)
{
    const int b = blockIdx.y;
    if (p.fresh[b] == 0) return;
    u32x4 *row = (u32x4 *)(p.seen + (int64_t)b * p.seen_row);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.seen_row / 8; i += (int64_t)gridDim.x * 256) row[i] = u32x4{0, 0, 0, 0};
}

__global__ __launch_bounds__(256) void count_tokens_kernel(const CountParams p)
{
    const int b = blockIdx.y;
    int len = p.lens[b];
    len = len < p.n ? len : p.n;
    const int prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
    uint32_t *row = (uint32_t *)(p.seen + (int64_t)b * p.seen_row);
    for (int i = blockIdx.x * 256 + threadIdx.x; i < len; i += gridDim.x * 256) {
        int at = i;
        if (p.path) {
            at = p.path[(int64_t)b * p.n + i];
            if (at < 0 || at >= p.n) continue;
        }
        const int x = p.tokens[(int64_t)b * p.n + at];
        if (x < 0 || x >= p.V) continue;
        uint32_t *word = row + (x >> 1);
        const int shift = (x & 1) * 16;
        if (i < prompt) {
            atomicOr(word, 0x8000u << shift);
            continue;
        }
        uint32_t old = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), then;
        do {
            if ((old >> shift & 0x7fff) == 0x7fff) break;
            then = old;
            old = atomicCAS(word, then, then + (1u << shift));
        } while (old != then);
    }
}

}  // namespace

// Slices of a row: 2,048 workgroups in all, as far as there are 2,048 tokens for each.
void probs_plan(ProbsParams &p)
{
    const int64_t rows = (int64_t)p.B * p.n;
    int64_t slices = (2048 + rows - 1) / rows;
    const int64_t most = ((int64_t)p.V + kStep - 1) / kStep, least = ((int64_t)p.V + kMostSlice - 1) / kMostSlice;
    if (slices > most) slices = most;
    if (slices < least) slices = least;
    p.slice_len = (int)(((p.V + slices - 1) / slices + kStep - 1) / kStep * kStep);
    p.slices = (int)(((int64_t)p.V + p.slice_len - 1) / p.slice_len);
    p.words = (int)(((int64_t)p.V + 31) / 32);
}

template <typename E>
static hipError_t launch_probs_t(const ProbsParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)p.B * p.n * p.slices));
    const size_t lds = p.masks || p.n_bias ? (size_t)(p.slice_len < p.V ? p.slice_len : p.V + 31) / 32 * 4 : 0;
    hipLaunchKernelGGL((token_stats_kernel<E>), grid, dim3(kThreads), lds, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((token_probs_kernel<E>), grid, dim3(kThreads), lds, stream, p);
    return hipGetLastError();
}

hipError_t launch_token_probs(const ProbsParams &p, int elem_bytes, hipStream_t stream)
{
    return elem_bytes == 2 ? launch_probs_t<uint16_t>(p, stream) : launch_probs_t<float>(p, stream);
}

hipError_t launch_count_tokens(const CountParams &p, hipStream_t stream)
{
    if (p.fresh) {
        const int64_t blocks = (p.seen_row / 8 + 255) / 256;
        hipLaunchKernelGGL(clear_seen_kernel, dim3((unsigned)(blocks < 64 ? blocks : 64), (unsigned)p.B), dim3(256), 0, stream, p);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const int blocks = (int)(((int64_t)p.n + 255) / 256);
    hipLaunchKernelGGL(count_tokens_kernel, dim3((unsigned)(blocks < 64 ? blocks : 64), (unsigned)p.B), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace loza
