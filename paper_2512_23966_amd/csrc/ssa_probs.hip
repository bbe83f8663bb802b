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
constexpr int kThreads = 256, kStep = kUnit * kThreads, kRowThreads = 512;
constexpr int kMostSlice = 131072;               // tokens of a slice (a bit each in LDS)
constexpr int kMostSpecial = kTreeNodes + kMostBias;

// What a row's logits are changed by
struct Change {
    float rep, fre, pre;
    // Each operation rounded by itself, as a plain program does them: a token next to another must not win by a rounding left out.
    __device__ __forceinline__ float operator()(float l, bool occurred, int said) const
    {
#pragma clang fp contract(off)
        const float up = l / rep, down = l * rep, was = occurred ? (l > 0.f ? up : down) : l, f = fre * (float)said, less = (was - f) - pre;
        return said > 0 ? less : was;
    }
};

// exp(d / T) for d <= 0: 2^(d c), c = log2(e) / T in two parts. Where a token does not weigh d is -infinity, or a NaN (nothing weighs yet): cut to what has a weight of 0.
struct Weight {
    float hi, lo, least;
    __device__ __forceinline__ explicit Weight(float t)
    {
        const double c = 1.4426950408889634074 / (double)t;
        hi = (float)c;
        lo = (float)(c - (double)hi);
        least = (float)(-200.0 / c);
    }
    // The rounding of the product left in (a sum of many: each off by 2^-24 of |d| / T, in either direction)
    __device__ __forceinline__ float rough(float d) const { return __builtin_amdgcn_exp2f(fmaxf(d, least) * hi); }
    // ... and given back to first order; times a factor
    __device__ __forceinline__ float exact(float d, float factor) const
    {
        const float x = fmaxf(d, least), h = x * hi, rest = __builtin_fmaf(x, lo, __builtin_fmaf(x, hi, -h)), p = __builtin_amdgcn_exp2f(h) * factor;
        return __builtin_fmaf(p * rest, 0.693147180559945f, p);
    }
};

// Largest logit, its first token, and the sum of the weights relative to it
struct Stat {
    float m, s;
    int32_t x, unused;
};
__device__ __forceinline__ void merge(Stat &a, float m, float s, int32_t x, const Weight &w)
{
    if (m == LOZA_NEG_INF) return;
    if (m > a.m) {
        a.s = s + a.s * w.rough(a.m - m);
        a.m = m;
        a.x = x;
    } else if (m == a.m) {                       // (two infinities among them)
        a.s += s;
        if (x < a.x) a.x = x;
    } else {
        a.s += s * w.rough(m - a.m);
    }
}

// -infinity in the place of a NaN. (A comparison: minimum and maximum would let signalling ones through, and a median of constants is folded to a minimum.)
__device__ __forceinline__ float settle(float l) { return l == l ? l : LOZA_NEG_INF; }

// Largest of a unit without NaNs (the instruction itself: for fmaxf the compiler first makes every operand quiet)
__device__ __forceinline__ float largest(const float (&l)[kUnit])
{
    float a, b;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(l[0]), "v"(l[1]), "v"(l[2]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(b) : "v"(l[3]), "v"(l[4]), "v"(l[5]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(a), "v"(l[6]), "v"(l[7]));
    return a > b ? a : b;
}

// What is read of 8 tokens
template <typename E>
struct Raw {
    u32x4 l[sizeof(E) / 2], z;
    uint32_t ok, apart;

    // The logits at `at`: rows of odd vocabularies are aligned to their elements only
    __device__ __forceinline__ void load(const E *at) { __builtin_memcpy(l, at, sizeof(l)); }
    __device__ __forceinline__ void load(const E *at, int n)         // n < 8 of them
    {
        E e[kUnit] = {};
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
            if (i < n) e[i] = at[i];
        __builtin_memcpy(l, e, sizeof(l));
    }
    __device__ __forceinline__ float logit(int i) const
    {
        // (named first: a bit cast of a vector's element itself takes its first one)
        const uint32_t x = sizeof(E) == 4 ? l[i / 4 % (sizeof(E) / 2)][i % 4] : i & 1 ? l[0][i / 2] & 0xffff0000u : l[0][i / 2] << 16;
        return __builtin_bit_cast(float, x);
    }
};

// One row's slice [x0, x1): the tokens that are done apart, and what the pass over the others needs.
template <typename E, int THREADS>
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
        for (int i = threadIdx.x; i < (x1 - x0 + 31) / 32; i += THREADS) bits[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < (entries + 3) / 4 * 4; i += THREADS) {
            int x = -1;
            if (i >= entries) {
            } else if (i < nodes) {
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
    // Everything of the tokens [x, x + 8) that is in memory; `whole`: all of them are there
    __device__ __forceinline__ void load(int x, bool whole, Raw<E> &raw) const
    {
        if (whole) raw.load(row + x);
        else raw.load(row + x, p.V - x);
        raw.z = u32x4{0, 0, 0, 0};
        if (seen) raw.z = *(const u32x4 *)(seen + x);
        raw.ok = 0xffu;
        if (allowed) raw.ok = allowed[x >> 3];
        if (!whole) raw.ok &= (1u << (p.V - x)) - 1;
        raw.apart = 0;
        if (entries) raw.apart = ((const uint8_t *)bits)[(x - x0) >> 3];
    }
    // Their changed logits; -inf for those done apart, not allowed, or not there
    __device__ __forceinline__ void changed(const Raw<E> &raw, float (&l)[kUnit]) const
    {
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = raw.logit(i);
        if (raw.z[0] | raw.z[1] | raw.z[2] | raw.z[3]) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) {
                const uint32_t z = i & 1 ? raw.z[i / 2] >> 16 : raw.z[i / 2] & 0xffffu;
                l[i] = change(l[i], z != 0, (int)(z & 0x7fffu));
            }
        }
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = settle(l[i]);
        const uint32_t ok = raw.ok & ~raw.apart;
        if (ok != 0xffu) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) {
                const uint32_t keep = (uint32_t)((int32_t)(ok << (31 - i)) >> 31), x = __builtin_bit_cast(uint32_t, l[i]);
                l[i] = __builtin_bit_cast(float, (x & keep) | (0xff800000u & ~keep));
            }
        }
    }
    // Calls f(x, raw, whole) for this thread's units, kAhead at a time so that their loads are under way together
    template <typename F>
    __device__ __forceinline__ void units(F f) const
    {
        constexpr int kAhead = sizeof(E) == 2 ? 2 : 1;
        int x = x0 + (int)threadIdx.x * kUnit;
        const int whole_end = (x1 - x0) / kUnit * kUnit + x0, step = THREADS * kUnit;
        for (; x + (kAhead - 1) * step < whole_end; x += kAhead * step) {
            Raw<E> raw[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) load(x + k * step, true, raw[k]);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) f(x + k * step, raw[k], true);
        }
        for (; x < whole_end; x += step) {
            Raw<E> raw;
            load(x, true, raw);
            f(x, raw, true);
        }
        if (x < x1) {                                                // (x is where the last, short unit begins, in one thread)
            Raw<E> raw;
            load(x, false, raw);
            f(x, raw, false);
        }
    }
    // The changed logit of entry i, and whether it is the one that stands for its token (the first of them)
    __device__ __forceinline__ bool special(int i, float &l) const
    {
#pragma clang fp contract(off)
        const int x = tok[i], nodes = p.masks ? p.n : 0;
        if (x < 0) return false;
        const int z = seen ? seen[x] : 0;
        int said = z & 0x7fff, first = i;
        float bias = 0.f;
        l = Elem<E>::get(row[x]);
        const bool ok = !allowed || (allowed[x >> 3] >> (x & 7) & 1);
#pragma unroll 2
        for (int k = 0; k < entries; k += 4) {                       // (behind the last entry there are -1)
            const i32x4 t = *(const i32x4 *)(tok + k);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t[j] == x) {
                    if (k + j < first) first = k + j;
                    if (k + j < nodes) ++said;
                    else bias = bias + p.bias_values[(int64_t)b * p.n_bias + k + j - nodes];
                }
        }
        if (first != i) return false;
        l = settle(change(l, z >= 0x8000 || said > 0, said) + bias);
        if (!ok) l = LOZA_NEG_INF;
        return true;
    }
};

// Requests whose temperature is 0 (or otherwise none to divide by) take the largest logit.
__device__ __forceinline__ float temperature_of(const ProbsParams &p, int b)
{
    const float t = p.temperature ? p.temperature[b] : 1.f;
    return t >= 0x1p-100f && t <= 0x1p100f ? t : 0.f;
}

// Stat of a whole workgroup, in all of its threads
template <int THREADS>
__device__ __forceinline__ Stat workgroup_stat(Stat a, const Weight &w, Stat *lds)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        // (the lower lane's first, in both of a pair: the same bits)
        const bool low = (threadIdx.x & d) == 0;
        const float m = __shfl_xor(a.m, d, 64), s = __shfl_xor(a.s, d, 64);
        const int x = __shfl_xor(a.x, d, 64);
        Stat first{low ? a.m : m, low ? a.s : s, low ? a.x : x, 0};
        merge(first, low ? m : a.m, low ? s : a.s, low ? x : a.x, w);
        a = first;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = lds[0];
    for (int i = 1; i < THREADS / 64; ++i) merge(a, lds[i].m, lds[i].s, lds[i].x, w);
    return a;
}

constexpr Stat kNoStat = {LOZA_NEG_INF, 0.f, 0x7fffffff, 0};

// Stat of this thread's share of a slice
template <typename E, int THREADS>
__device__ __forceinline__ Stat thread_stat(const Slice<E, THREADS> &s, float t, const Weight &w)
{
    Stat a = kNoStat;
    s.units([&](int x, const Raw<E> &raw, bool) {
        float l[kUnit];
        s.changed(raw, l);
        const float m = largest(l);
        if (m > a.m) {
            a.s *= w.rough(a.m - m);
            a.m = m;
            if (!(t > 0.f)) {
                int at = 0;
#pragma unroll
                for (int i = kUnit - 1; i >= 0; --i) at = l[i] == m ? i : at;
                a.x = x + at;
            }
        }
        if (t > 0.f && a.m < __builtin_inff()) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) a.s += w.rough(l[i] - a.m);
        } else if (t > 0.f) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) a.s += l[i] == a.m ? 1.f : 0.f;     // (those of +infinity share the row)
        }
    });
    for (int i = threadIdx.x; i < s.entries; i += THREADS) {
        float l;
        if (s.special(i, l)) merge(a, l, 1.f, s.tok[i], w);
    }
    return a;
}

// The probabilities of a slice, given the Stat of its row
template <typename E, int THREADS>
__device__ __forceinline__ void write_probs(const Slice<E, THREADS> &s, float *out, const Stat &a, float t, const Weight &w)
{
    const bool greedy = !(t > 0.f);
    const float inv = a.m == LOZA_NEG_INF ? 0.f : 1.f / a.s;
    const bool infinite = a.m == __builtin_inff();
    auto prob = [&](float l, int x) { return greedy ? (x == a.x ? 1.f : 0.f) : infinite ? (l == a.m ? inv : 0.f) : w.exact(l - a.m, inv); };
    s.units([&](int x, const Raw<E> &raw, bool whole) {
        float l[kUnit];
        s.changed(raw, l);
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = prob(l[i], x + i);
        if (raw.apart == 0 && whole) {
            __builtin_memcpy(out + x, l, sizeof(l));
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i)
                if (!(raw.apart >> i & 1) && x + i < s.p.V) out[x + i] = l[i];
        }
    });
    for (int i = threadIdx.x; i < s.entries; i += THREADS) {
        float l;
        if (s.special(i, l)) out[s.tok[i]] = prob(l, s.tok[i]);
    }
}

// Whether a row is one of its tree's
__device__ __forceinline__ bool row_there(const ProbsParams &p, int64_t row)
{
    return p.tree_lens == nullptr || (int)(row % p.n) < p.tree_lens[row / p.n];
}

template <typename E>
__global__ __launch_bounds__(kThreads) void token_stats_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ __attribute__((aligned(16))) int32_t s_tok[kMostSpecial];
    __shared__ Stat s_stat[kThreads / 64];
    const int64_t row = blockIdx.x / p.slices;
    if (!row_there(p, row)) return;
    const Slice<E, kThreads> s(p, row, (int)(blockIdx.x - row * p.slices), s_tok, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    const Stat a = workgroup_stat<kThreads>(thread_stat(s, t, w), w, s_stat);
    if (threadIdx.x == 0) ((Stat *)p.stats)[blockIdx.x] = a;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void token_probs_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ __attribute__((aligned(16))) int32_t s_tok[kMostSpecial];
    __shared__ Stat s_stat[kThreads / 64];
    const int64_t row = blockIdx.x / p.slices;
    if (!row_there(p, row)) return;
    const Slice<E, kThreads> s(p, row, (int)(blockIdx.x - row * p.slices), s_tok, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    Stat a = kNoStat;
    for (int i = threadIdx.x; i < p.slices; i += kThreads) {
        const Stat part = ((const Stat *)p.stats)[row * p.slices + i];
        merge(a, part.m, part.s, part.x, w);
    }
    a = workgroup_stat<kThreads>(a, w, s_stat);
    write_probs(s, p.probs + row * p.V, a, t, w);
}

// A workgroup a row, in one launch: the row is read again for the probabilities, from a cache that holds what is under way.
template <typename E>
__global__ __launch_bounds__(kRowThreads) void token_row_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ __attribute__((aligned(16))) int32_t s_tok[kMostSpecial];
    __shared__ Stat s_stat[kRowThreads / 64];
    const int64_t row = blockIdx.x;
    if (!row_there(p, row)) return;
    const Slice<E, kRowThreads> s(p, row, 0, s_tok, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    const Stat a = workgroup_stat<kRowThreads>(thread_stat(s, t, w), w, s_stat);
    write_probs(s, p.probs + row * p.V, a, t, w);
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

// The same for many tokens: a workgroup takes a slice of a request's row, counts in LDS (bit 31: in the prompt) what of all tokens falls into it, and
// writes the units of 8 that changed. Every slice reads all tokens, out of L2.
constexpr int kCountSlice = 16384, kCountThreads = 1024;

__global__ __launch_bounds__(kCountThreads) void count_slice_kernel(const CountParams p)
{
    __shared__ uint32_t s_count[kCountSlice];
    const int b = blockIdx.y, x0 = blockIdx.x * kCountSlice;
    for (int i = threadIdx.x; i < kCountSlice; i += kCountThreads) s_count[i] = 0;
    __syncthreads();
    int len = p.lens[b];
    len = len < p.n ? len : p.n;
    const int prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
    const int32_t *tokens = p.tokens + (int64_t)b * p.n, *path = p.path ? p.path + (int64_t)b * p.n : nullptr;
    const uint32_t end = (uint32_t)(x0 >= p.V ? 0 : p.V - x0 < kCountSlice ? p.V - x0 : kCountSlice);     // (a row may be longer than the vocabulary)
    auto note = [&](int i, int x) {
        const uint32_t at = (uint32_t)(x - x0);                      // (tokens outside the slice, negative ones too, are large)
        if (x < x0 || at >= end) return;
        if (i < prompt) atomicOr(&s_count[at], 0x80000000u);
        else atomicAdd(&s_count[at], 1u);                            // (fewer than 2^31 of them)
    };
    if (path) {
        for (int i = threadIdx.x; i < len; i += kCountThreads) {
            const int at = path[i];
            if (at >= 0 && at < p.n) note(i, tokens[at]);
        }
    } else {
#pragma unroll 4
        for (int i = threadIdx.x * 4; i < len; i += kCountThreads * 4) {
            if (i + 4 <= len) {
                i32x4 x;
                __builtin_memcpy(&x, tokens + i, 16);                // (rows of odd lengths are aligned to their elements only)
#pragma unroll
                for (int k = 0; k < 4; ++k) note(i + k, x[k]);
            } else {
                for (int k = i; k < len; ++k) note(k, tokens[k]);
            }
        }
    }
    __syncthreads();
    const bool fresh = p.fresh && p.fresh[b] != 0;
    uint16_t *row = p.seen + (int64_t)b * p.seen_row;
    for (int i = threadIdx.x * 8; i < kCountSlice; i += kCountThreads * 8) {
        if ((int64_t)x0 + i >= p.seen_row) break;
        uint32_t any = 0, c[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) any |= c[k] = s_count[i + k];
        if (!any && !fresh) continue;
        Pack<uint16_t, 8> z{};
        if (!fresh) z = *(const Pack<uint16_t, 8> *)(row + x0 + i);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t said = (z.e[k] & 0x7fffu) + (c[k] & 0x7fffffffu);
            z.e[k] = (uint16_t)((said < 0x7fffu ? said : 0x7fffu) | (z.e[k] & 0x8000u) | (c[k] >> 31 << 15));
        }
        *(Pack<uint16_t, 8> *)(row + x0 + i) = z;
    }
}

}  // namespace

constexpr int kRows = 256;

// Slices of a row: 2,048 workgroups in all, as far as there are 2,048 tokens for each.
void probs_plan(ProbsParams &p)
{
    const int64_t rows = (int64_t)p.B * p.n;
    int64_t slices = rows >= kRows ? 1 : (2048 + rows - 1) / rows;
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
    if (p.slices == 1 && p.V > kStep) {
        hipLaunchKernelGGL((token_row_kernel<E>), grid, dim3(kRowThreads), lds, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((token_stats_kernel<E>), grid, dim3(kThreads), lds, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((token_probs_kernel<E>), grid, dim3(kThreads), lds, stream, p);
    return hipGetLastError();
}

hipError_t launch_token_probs(const ProbsParams &p, int elem_bytes, hipStream_t stream)
{
    return elem_bytes == 2 ? launch_probs_t<uint16_t>(p, stream) : launch_probs_t<float>(p, stream);
}

constexpr int kManyTokens = 1024;

hipError_t launch_count_tokens(const CountParams &p, hipStream_t stream)
{
    const int64_t slices = (p.seen_row + kCountSlice - 1) / kCountSlice;
    if (p.n >= kManyTokens && slices <= 64) {
        hipLaunchKernelGGL(count_slice_kernel, dim3((unsigned)slices, (unsigned)p.B), dim3(kCountThreads), 0, stream, p);
        return hipGetLastError();
    }
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
