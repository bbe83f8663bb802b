// Probabilities of the next token from logits, under penalties for repeated tokens, biases and grammar masks (gfx950), and the
// record of a request's tokens that the penalties read.
//
// Token x of a row has the logit l, the number c of times it was said and whether it occurred at all (said, or in the prompt):
//     l' = l / repetition if l > 0, l * repetition otherwise, where it occurred;  l'' = l' - frequency c - presence (c > 0) + bias
// and no weight where the grammar does not allow it (or l'' is a NaN); p = exp((l'' - max) / T) / sum, or 1 at the first of the largest.
//
// What bounds it: memory without penalties, 4 bytes a token out and 2 or 4 in (1,024 rows of 131,072 bf16 logits 169 us, 4.8 TB/s, fp32 251, 4.3 TB/s); with everything the vector ALU
// as well, 39 instructions a token in two passes (bf16, 853 of the rows alive: 210 us, 159 where a cache has the logits; the memory's part is 136). All of it is done
// on the way. The tokens of a tree's own nodes and the biased ones are a few hundred of 100,000: the pass over the row leaves
// them out (a bit each in LDS), and a thread each does them apart, so that the pass looks nothing up.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_rope.h"
#include "ssa_step.h"

namespace loza {

namespace {

// A wave takes 512 tokens at a time, a lane 4 of the first half and 4 of the second: so its two stores of 16 bytes lie side by side with its neighbours'. (Of 8
// tokens in a row it would be 16 bytes of every 32: 670 MB in and out 179 us, with halves 147.)
constexpr int kUnit = 8, kHalf = 256, kBlock = 2 * kHalf;
__device__ __forceinline__ constexpr int token_of(int x, int i) { return x + (i & 3) + (i >> 2) * kHalf; }     // token i of a lane whose first is x
constexpr int kThreads = 256, kStep = kUnit * kThreads;
constexpr int kMostSlice = 262144;               // tokens of a slice (a bit each in LDS; 768 rows of 200,064, us: 263, with two slices each 311)
constexpr int kMostSpecial = kTreeNodes + kMostBias;

// What a row's logits are changed by. Where the largest is asked for (greedy rows) each operation is rounded by itself, as a plain program does them: a token
// next to another must not win by a rounding left out. Elsewhere (`soft`) a few units do not matter, and half of the instructions do.
struct Change {
    float rep, inv, inv_lo, fre, pre;  // inv + inv_lo: 1 / rep
    bool quick;                        // the division by `rep` as below (and what is said of small quotients there)
    bool repeats, counts, occurs;      // which of the three change anything: requests rarely ask for all of them (853 rows of 131,072, a sixth of them said: 215 -> 196 us)

    __device__ __forceinline__ void set(float rep_, float fre_, float pre_)
    {
        rep = rep_;
        inv = 1.f / rep_;
        inv_lo = __builtin_fmaf(-inv, rep_, 1.f) * inv;
        fre = fre_;
        pre = pre_;
        quick = rep >= 0x1p-20f && rep <= 0x1p20f && (fre_ == 0.f || fabsf(fre_) >= 0x1p-50f);
        repeats = rep_ != 1.f;
        counts = fre_ != 0.f;
        occurs = pre_ != 0.f || !(fabsf(fre_) < __builtin_inff());   // (infinity times 0 is not 0)
    }
    __device__ __forceinline__ float soft(float l, bool occurred, uint32_t said) const
    {
        const float less = said != 0 ? __builtin_fmaf(fre, (float)said, pre) : 0.f;
        return __builtin_fmaf(l, factor(l, occurred), -less);
    }
    __device__ __forceinline__ float factor(float l, bool occurred) const
    {
        const float f = l > 0.f ? inv : rep;
        return occurred ? f : 1.f;
    }
    // The same of a lane's tokens, z(i) the record of the i-th
    template <typename F>
    __device__ __forceinline__ void soft(float (&l)[kUnit], F z) const
    {
        float less[kUnit] = {};
        if (!occurs) {
            if (counts) {
#pragma unroll
                for (int i = 0; i < kUnit; ++i) less[i] = fre * (float)(z(i) & 0x7fffu);
            }
        } else if (!counts) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) less[i] = (z(i) & 0x7fffu) != 0 ? pre : 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) less[i] = (z(i) & 0x7fffu) != 0 ? __builtin_fmaf(fre, (float)(z(i) & 0x7fffu), pre) : 0.f;
        }
        if (repeats) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] = __builtin_fmaf(l[i], factor(l[i], z(i) != 0), -less[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] -= less[i];
        }
    }
    __device__ __forceinline__ float rounded(float l, bool occurred, uint32_t said) const
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
    // The same without branches of lanes. l / rep as l (inv + inv_lo), which is off by less than a unit, and a correction by what is left, fma(-q, rep, l) inv: that gives
    // the rounded quotient (Markstein 1990) where what is left is exact, which takes l and q of 2^-100 and more; with the repetitions that are `quick` a q of 2^-80 and more
    // has both (smaller ones: small_matters). One that overflows comes out as a NaN.
    template <typename F>
    __device__ __forceinline__ void quickly(float (&l)[kUnit], F z) const
    {
#pragma clang fp contract(off)
        if (repeats) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) {
                float q = __builtin_fmaf(l[i], inv_lo, l[i] * inv);
                q = __builtin_fmaf(__builtin_fmaf(-q, rep, l[i]), inv, q);
                const float r = __builtin_amdgcn_classf(l[i], 0x180) ? q : l[i] * rep;         // (positive and finite)
                l[i] = z(i) != 0 ? r : l[i];
            }
        }
        if (counts) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) {
                const float f = fre * (float)(z(i) & 0x7fffu);       // (0 where the token was not said)
                l[i] -= f;
            }
        }
        if (occurs) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] -= (z(i) & 0x7fffu) != 0 ? pre : 0.f;
        }
    }
    // Whether quotients of less than 2^-80, which may be off by a step, can decide which of a lane's tokens is the largest: not next to one of 2^-50 or more, before them or
    // among them, nor where all are at -2^-50 or below. A penalty of 2^-50 or more leaves of them what it leaves of 0, and what a smaller one leaves is smaller than 2^-50.
    __device__ __forceinline__ bool small_matters(float before, float largest) const { return before < 0x1p-50f && fabsf(largest) < 0x1p-50f; }
};

// exp(d / T) for d <= 0: 2^(d c), c = log2(e) / T. -infinity gives 0. Off by 2^-24 of |d| / T twice (the product, and c) and by the exponential's own unit.
struct Weight {
    float c;
    __device__ __forceinline__ explicit Weight(float t) : c((float)(1.4426950408889634074 / (double)t)) {}
    __device__ __forceinline__ float operator()(float d) const { return __builtin_amdgcn_exp2f(d * c); }
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
        a.s = s + a.s * w(a.m - m);
        a.m = m;
        a.x = x;
    } else if (m == a.m) {                       // (two infinities among them)
        a.s += s;
        if (x < a.x) a.x = x;
    } else {
        a.s += s * w(m - a.m);
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

// Requests whose temperature is 0 (or otherwise none to divide by) take the largest logit.
__device__ __forceinline__ float temperature_of(const ProbsParams &p, int b)
{
    const float t = p.temperature ? p.temperature[b] : 1.f;
    return t >= 0x1p-100f && t <= 0x1p100f ? t : 0.f;
}

// What is read of a lane's 8 tokens
template <typename E>
struct Raw {
    static constexpr int kWords = 4 * sizeof(E) / 4;                 // of a half
    uint32_t l[2 * kWords], z[4], ok;

    __device__ __forceinline__ float logit(int i) const
    {
        const uint32_t x = sizeof(E) == 4 ? l[i % (2 * kWords)] : i & 1 ? l[i / 2] & 0xffff0000u : l[i / 2] << 16;
        return __builtin_bit_cast(float, x);
    }
    __device__ __forceinline__ uint32_t record(int i) const { return i & 1 ? z[i / 2] >> 16 : z[i / 2] & 0xffffu; }
};

// (not fused with what comes before)
__device__ __forceinline__ float add(float a, float b)
{
#pragma clang fp contract(off)
    return a + b;
}

// The tokens that are done apart, in LDS: those of a block of 512 as a list from first[block] on, -1 at its end
struct Special {
    int32_t tok[kMostSpecial], again;
    float val[kMostSpecial];
    int32_t first[kMostSlice / kBlock], next[kMostSpecial];
};

// kPlain: no tokens that are done apart, no record and no grammar; kNoRecord: no record. (Kernels of their own: a wait for what a wave has asked for counts the loads behind it,
// and with loads that may be there or not it is for all of them.)
constexpr int kPlain = 0, kNoRecord = 1, kRecord = 2;

// One row's slice [x0, x1): the tokens that are done apart, and what the pass over the others needs.
template <typename E, int THREADS, int KIND>
struct Slice {
    const ProbsParams &p;
    const E *row;
    const uint16_t *seen;
    const uint8_t *allowed;
    int b, r, x0, x1, entries;
    uint32_t bits_mine = 0;       // which of this thread's entries stand for their tokens (1,088 entries are at most 5 a thread)
    Change change;
    bool soft;
    Special &lds;                 // tok: tokens done apart, -1 where they are not in the slice; val: their changed logits
    uint32_t *bits;               // LDS: a bit a token of the slice: done apart, or not allowed

    __device__ __forceinline__ Slice(const ProbsParams &p_, int64_t row_index, int slice, Special &lds_, uint32_t *bits_) : p(p_), lds(lds_), bits(bits_)
    {
        b = (int)(row_index / p.n);
        r = (int)(row_index - (int64_t)b * p.n);
        row = (const E *)p.logits + row_index * p.logits_row;
        seen = p.seen ? p.seen + (int64_t)b * p.seen_row : nullptr;
        allowed = p.allowed ? (const uint8_t *)(p.allowed + row_index * p.words) : nullptr;
        x0 = slice * p.slice_len;
        x1 = x0 + p.slice_len < p.V ? x0 + p.slice_len : p.V;
        if constexpr (KIND == kPlain) {
            entries = 0;
            return;
        }
        change.set(p.repetition ? p.repetition[b] : 1.f, p.frequency ? p.frequency[b] : 0.f, p.presence ? p.presence[b] : 0.f);
        soft = temperature_of(p, b) > 0.f;
        const int nodes = p.masks ? p.n : 0;
        entries = nodes + p.n_bias;
        const int words = (x1 - x0 + 31) / 32;
        if (entries == 0) {
            bar(words);
            return;
        }
        uint64_t path = nodes ? (uint64_t)p.masks[row_index] : 0;    // (nodes before the tree's end)
        if (nodes) path &= length() >= 64 ? ~0ull : (1ull << (length() > 0 ? length() : 0)) - 1;
        for (int i = threadIdx.x; i < words; i += THREADS) bits[i] = 0;
        for (int i = threadIdx.x; i < (x1 - x0 + kBlock - 1) / kBlock; i += THREADS) lds.first[i] = -1;
        if (threadIdx.x == 0) lds.again = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < entries; i += THREADS) {
            int x = i < nodes ? p.tokens[(int64_t)b * p.n + i] : p.bias_tokens[(int64_t)b * p.n_bias + i - nodes];
            if (x < x0 || x >= x1 || (i < nodes && !(path >> i & 1))) x = -1;
            lds.tok[i] = x;
            if (x >= 0) {
                const uint32_t bit = 1u << ((x - x0) & 31);
                if (atomicOr(&bits[(x - x0) >> 5], bit) & bit) lds.again = 1;
            }
        }
        __syncthreads();
        // their logits; a token that is there more than once is done by the first of its entries
        const bool again = lds.again != 0;
        for (int i = threadIdx.x; i < entries; i += THREADS) {
            float l = 0.f;
            const bool mine = special(i, again, l);
            lds.val[i] = l;
            if (mine) bits_mine |= 1u << (i / THREADS);
        }
        if (again) __syncthreads();                                   // (all have looked at the tokens)
        for (int i = threadIdx.x; i < entries; i += THREADS) {
            if (bits_mine >> (i / THREADS) & 1) lds.next[i] = atomicExch(&lds.first[(lds.tok[i] - x0) / kBlock], i);
            else lds.tok[i] = -1;
        }
        bar(words);
    }
    // Adds the tokens that are not allowed to the bits
    __device__ __forceinline__ void bar(int words)
    {
        if (allowed == nullptr) return;
        const uint32_t *from = (const uint32_t *)allowed + x0 / 32;
        for (int i = threadIdx.x; i < words; i += THREADS) bits[i] = (entries ? bits[i] : 0u) | ~from[i];
        __syncthreads();
    }
    __device__ __forceinline__ int length() const
    {
        const int len = p.tree_lens ? p.tree_lens[b] : p.n;
        return len < p.n ? len : p.n;
    }
    // Everything of a lane's tokens that is in memory; `whole`: the wave's are all there
    __device__ __forceinline__ void load(int x, bool whole, Raw<E> &raw) const
    {
        constexpr int W = Raw<E>::kWords;
        raw.ok = ok_of(x, whole);
        if (KIND != kPlain && whole && !__any(raw.ok != 0)) x = 4 * (threadIdx.x & 63) + x0;         // (none of 512 tokens is allowed: something that a cache has)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int xh = x + h * kHalf;
            raw.z[2 * h] = raw.z[2 * h + 1] = 0;
            if (whole) {
                __builtin_memcpy(raw.l + h * W, row + xh, 4 * sizeof(E));      // (rows of odd vocabularies are aligned to their elements only)
            } else {                                                           // tokens that are not there: the last one again
                E e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = row[xh + i < p.V ? xh + i : p.V - 1];
                __builtin_memcpy(raw.l + h * W, e, sizeof(e));
            }
            if constexpr (KIND == kRecord) {
                const u32x2 z = *(const u32x2 *)(seen + (whole || xh < p.V ? xh : (p.V - 1) & ~3));
                raw.z[2 * h] = z[0];
                raw.z[2 * h + 1] = z[1];
            }
        }
    }
    // Which of a lane's tokens are there, allowed and not done apart
    __device__ __forceinline__ uint32_t ok_of(int x, bool whole) const
    {
        uint32_t all = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int xh = x + h * kHalf, n = whole ? 4 : p.V - xh;
            if (n <= 0) continue;
            uint32_t ok = 15u;
            if (KIND != kPlain && (entries || allowed)) ok = ~((uint32_t)((const uint8_t *)bits)[(xh - x0) >> 3] >> (xh & 4)) & 15u;
            if (!whole && n < 4) ok &= (1u << n) - 1;
            all |= ok << (4 * h);
        }
        return all;
    }
    // Their changed logits; -inf for those done apart, not allowed, or not there
    template <bool SOFT>
    __device__ __forceinline__ void changed(int x, bool whole, const Raw<E> &raw, float (&l)[kUnit]) const
    {
        if (KIND != kPlain && !__any(raw.ok != 0)) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] = LOZA_NEG_INF;
            return;
        }
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = raw.logit(i);
        // (branches of whole waves: a branch of lanes has the compiler keep a copy of everything)
        bool again = false;
        if (KIND == kRecord && __any((raw.z[0] | raw.z[1] | raw.z[2] | raw.z[3]) != 0)) {
            auto z = [&](int i) { return raw.record(i); };
            if constexpr (SOFT) change.soft(l, z);
            else change.quickly(l, z);
            again = !SOFT && !change.quick;
        }
        // (two a comparison, in scalar registers: as a condition of lanes it is 16 instructions)
        uint64_t nans = 0;
#pragma unroll
        for (int i = 0; i < kUnit; i += 2) nans |= __builtin_amdgcn_ballot_w64(__builtin_isunordered(l[i], l[i + 1]));
        if (again || nans) {
            if (KIND == kPlain || SOFT) {
#pragma unroll
                for (int i = 0; i < kUnit; ++i) l[i] = settle(l[i]);
            } else {
                once_more(x, l);
            }
        }
        if (KIND != kPlain || !whole) bar_tokens(raw, l);
    }
    // The changed logits of a lane's tokens from memory, so that nothing is kept for this: NaNs, and quotients that are not sure
    __device__ __forceinline__ void once_more(int x, float (&l)[kUnit]) const
    {
#pragma unroll 1
        for (int i = 0; i < kUnit; ++i) {
            const int xi = token_of(x, i);
            float y = LOZA_NEG_INF;
            if (xi < p.V) {
                const uint32_t z = seen ? seen[xi] : 0u;
                y = settle(change.rounded(Elem<E>::get(row[xi]), z != 0, z & 0x7fffu));
            }
#pragma unroll
            for (int k = 0; k < kUnit; ++k) l[k] = k == i ? y : l[k];
        }
    }
    // -inf for tokens done apart, not allowed, or not there
    __device__ __forceinline__ static void bar_tokens(const Raw<E> &raw, float (&l)[kUnit])
    {
        if (!__any(raw.ok != 0xffu)) return;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) {
            const uint32_t keep = (uint32_t)((int32_t)(raw.ok << (31 - i)) >> 31), y = __builtin_bit_cast(uint32_t, l[i]);
            l[i] = __builtin_bit_cast(float, (y & keep) | (0xff800000u & ~keep));
        }
    }
    // Calls f(x, raw, whole) for this wave's blocks of 512 tokens; the next one's loads are under way meanwhile
    template <typename F>
    __device__ __forceinline__ void units(F f) const
    {
        constexpr int step = THREADS * kUnit;
        const int lane4 = 4 * (threadIdx.x & 63);
        int at = x0 + (int)(threadIdx.x >> 6) * kBlock;              // the block's first token
        Raw<E> raw[2];
        auto there = [&](int y) { return y + kBlock <= x1; };
        if (there(at)) {
            load(at + lane4, true, raw[0]);
            for (;;) {
                // (behind the last one the same again: always as many loads)
                load((there(at + step) ? at + step : at) + lane4, true, raw[1]);
                f(at + lane4, raw[0], true);
                at += step;
                if (!there(at)) break;
                load((there(at + step) ? at + step : at) + lane4, true, raw[0]);
                f(at + lane4, raw[1], true);
                at += step;
                if (!there(at)) break;
            }
        }
        for (; at < x1; at += step) {
            load(at + lane4, false, raw[0]);
            f(at + lane4, raw[0], false);
        }
    }
    // An entry of a list, the same for the whole wave
    __device__ __forceinline__ static int list(const int32_t *of, int i) { return __builtin_amdgcn_readfirstlane(of[i]); }
    // The changed logit of entry i, and whether it is the one that stands for its token; `again`: some token is there more than once
    __device__ __forceinline__ bool special(int i, bool again, float &l) const
    {
        const int x = lds.tok[i], nodes = p.masks ? p.n : 0;
        if (x < 0) return false;
        const int z = seen ? seen[x] : 0;
        const bool ok = !allowed || (allowed[x >> 3] >> (x & 7) & 1);
        const float *values = p.bias_values + (int64_t)b * p.n_bias;
        int said = z & 0x7fff, first = i;
        float bias = 0.f;
        l = Elem<E>::get(row[x]);
        if (!again) {
            if (i < nodes) ++said;
            else bias = values[i - nodes];
        } else {
#pragma unroll 8
            for (int k = 0; k < entries; ++k) {
                if (lds.tok[k] != x) continue;
                if (k < first) first = k;
                if (k < nodes) ++said;
                else bias = add(bias, values[k - nodes]);
            }
        }
        const bool occurred = z >= 0x8000 || said > 0;
        l = soft ? change.soft(l, occurred, (uint32_t)said) : change.rounded(l, occurred, (uint32_t)said);
        l = settle(add(l, bias));
        if (!ok) l = LOZA_NEG_INF;
        return first == i;
    }
};

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
template <bool SOFT, typename E, int THREADS, int KIND>
__device__ __forceinline__ Stat thread_stat_t(const Slice<E, THREADS, KIND> &s, const Weight &w)
{
    Stat a = kNoStat;
    s.units([&](int x, const Raw<E> &raw, bool whole) {
        float l[kUnit];
        s.template changed<SOFT>(x, whole, raw, l);
        float m = largest(l);
        if constexpr (!SOFT && KIND == kRecord) {
            if (s.change.repeats && __any(s.change.small_matters(a.m, m))) {
                s.once_more(x, l);
                s.bar_tokens(raw, l);
                m = largest(l);
            }
        }
        if (m > a.m) {
            if constexpr (SOFT) {
                a.s *= w(a.m - m);
            } else {
                int at = 0;
#pragma unroll
                for (int i = kUnit - 1; i >= 0; --i) at = l[i] == m ? token_of(0, i) : at;
                a.x = x + at;
            }
            a.m = m;
        }
        if constexpr (SOFT) {
            if (a.m > LOZA_NEG_INF && a.m < __builtin_inff()) {
#pragma unroll
                for (int i = 0; i < kUnit; ++i) a.s += w(l[i] - a.m);
            } else if (a.m > 0.f) {
#pragma unroll
                for (int i = 0; i < kUnit; ++i) a.s += l[i] == a.m ? 1.f : 0.f;     // (those of +infinity share the row)
            }
        }
    });
    if constexpr (KIND != kPlain)
        for (int i = threadIdx.x; i < s.entries; i += THREADS)
            if (s.lds.tok[i] >= 0) merge(a, s.lds.val[i], 1.f, s.lds.tok[i], w);
    return a;
}

// 8 results of a lane. (Two stores written out: one in either branch of a condition is merged to a plain one.)
template <bool NT>
__device__ __forceinline__ void store_unit(float *out, int x, int V, bool whole, const float (&l)[kUnit])
{
    if (whole) {
        typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
        u32x4 y[2];
        __builtin_memcpy(y, l, sizeof(y));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if constexpr (NT) __builtin_nontemporal_store(y[k], (u32x4_at4 *)(out + x + kHalf * k));
            else *(u32x4_at4 *)(out + x + kHalf * k) = y[k];
        }
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
            if (token_of(x, i) < V) out[token_of(x, i)] = l[i];
    }
}

// The probabilities of a slice of a row that is not greedy, given the row's Stat
template <bool NT, typename E, int THREADS, int KIND>
__device__ __forceinline__ void write_soft(const Slice<E, THREADS, KIND> &s, float *out, const Stat &a, const Weight &w)
{
    const float inv = a.m == LOZA_NEG_INF ? 0.f : 1.f / a.s;
    const bool infinite = a.m == __builtin_inff() || a.m == LOZA_NEG_INF;       // (nothing weighs: 0 for all)
    auto rare = [&](float l) { return l == a.m ? inv : 0.f; };
    s.units([&](int x, const Raw<E> &raw, bool whole) {
        float l[kUnit];
        s.template changed<true>(x, whole, raw, l);
        if (infinite) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] = rare(l[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) l[i] = w(l[i] - a.m) * inv;
        }
        if (KIND != kPlain && s.entries) {
            // those done apart, into what is stored (single words behind it took 10 us of 170 for 64 of them in each of 853 rows)
            for (int e = s.list(s.lds.first, (x - s.x0) / kBlock); e >= 0; e = s.list(s.lds.next, e)) {
                const int at = s.lds.tok[e] - x;
                const float y = infinite ? rare(s.lds.val[e]) : w(s.lds.val[e] - a.m) * inv;
#pragma unroll
                for (int i = 0; i < kUnit; ++i) l[i] = at == token_of(0, i) ? y : l[i];
            }
        }
        store_unit<NT>(out, x, s.p.V, whole, l);
    });
}

// ... of tokens [x0, x1) of a greedy one: nothing is read again
template <bool NT, int THREADS>
__device__ __forceinline__ void write_greedy(float *out, int x0, int x1, int V, int32_t first)
{
    for (int at = x0 + (int)(threadIdx.x >> 6) * kBlock; at < x1; at += THREADS * kUnit) {
        const int x = at + 4 * (threadIdx.x & 63);
        float l[kUnit];
#pragma unroll
        for (int i = 0; i < kUnit; ++i) l[i] = token_of(x, i) == first ? 1.f : 0.f;
        store_unit<NT>(out, x, V, at + kBlock <= x1, l);
    }
}

template <typename E, int THREADS, int KIND>
__device__ __forceinline__ Stat thread_stat(const Slice<E, THREADS, KIND> &s, float t, const Weight &w)
{
    return t > 0.f ? thread_stat_t<true>(s, w) : thread_stat_t<false>(s, w);
}
// Whether a row is one of its tree's
__device__ __forceinline__ bool row_there(const ProbsParams &p, int64_t row)
{
    return p.tree_lens == nullptr || (int)(row % p.n) < p.tree_lens[row / p.n];
}

template <typename E, int KIND>
__global__ __launch_bounds__(kThreads) void token_stats_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ Special s_special;
    __shared__ Stat s_stat[kThreads / 64];
    const int64_t row = blockIdx.x / p.slices;
    if (!row_there(p, row)) return;
    const Slice<E, kThreads, KIND> s(p, row, (int)(blockIdx.x - row * p.slices), s_special, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    const Stat a = workgroup_stat<kThreads>(thread_stat(s, t, w), w, s_stat);
    if (threadIdx.x == 0) ((Stat *)p.stats)[blockIdx.x] = a;
}

template <typename E, int KIND, bool NT>
__global__ __launch_bounds__(kThreads) void token_probs_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ Special s_special;
    __shared__ Stat s_stat[kThreads / 64];
    const int64_t row = blockIdx.x / p.slices;
    if (!row_there(p, row)) return;
    const int slice = (int)(blockIdx.x - row * p.slices);
    const float t = temperature_of(p, (int)(row / p.n));
    const Weight w(t > 0.f ? t : 1.f);
    float *out = p.probs + row * p.V;
    const Stat *parts = (const Stat *)p.stats + row * p.slices;
    Stat a = kNoStat;
    if ((int)threadIdx.x < p.slices) a = parts[threadIdx.x];
    auto stat = [&]() {
        for (int i = threadIdx.x + kThreads; i < p.slices; i += kThreads) merge(a, parts[i].m, parts[i].s, parts[i].x, w);
        return workgroup_stat<kThreads>(a, w, s_stat);
    };
    if (t > 0.f) {
        const Slice<E, kThreads, KIND> s(p, row, slice, s_special, s_bits);
        write_soft<NT>(s, out, stat(), w);
    } else {
        const int x0 = slice * p.slice_len;
        write_greedy<NT, kThreads>(out, x0, x0 + p.slice_len < p.V ? x0 + p.slice_len : p.V, p.V, stat().x);
    }
}

// A workgroup a row, in one launch: the row is read again for the probabilities, from a cache that holds what is under way.
template <typename E, int THREADS, int KIND, bool NT>
__global__ __launch_bounds__(THREADS) void token_row_kernel(const ProbsParams p)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_bits[];
    __shared__ Special s_special;
    __shared__ Stat s_stat[THREADS / 64];
    const int64_t row = blockIdx.x;
    if (!row_there(p, row)) return;
    const Slice<E, THREADS, KIND> s(p, row, 0, s_special, s_bits);
    const float t = temperature_of(p, s.b);
    const Weight w(t > 0.f ? t : 1.f);
    const Stat a = workgroup_stat<THREADS>(thread_stat(s, t, w), w, s_stat);
    float *out = p.probs + row * p.V;
    if (t > 0.f) write_soft<NT>(s, out, a, w);
    else write_greedy<NT, THREADS>(out, 0, p.V, p.V, a.x);
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
// writes the units of 8 that changed. Every slice reads all tokens, four loads of four under way (16 requests of 100,000 tokens 12.4 us, 14.5 with slices of 16,384, 19.5 with a load
// at a time). That reading is what it takes: 10.5 us without the comparisons and the counting, 11.0 with the comparisons. Each request's slices lie on all 8 dies, so each die's L2 (4 MB)
// asks for the 6.4 MB of all requests, 55 MB in all, and half of the 875,000 requests to L2 miss. How the tokens are spread does not show (evenly, or half of them in one slice: 12.4).
constexpr int kCountSlice = 8192, kCountThreads = 1024;

__global__ __launch_bounds__(kCountThreads) void count_slice_kernel(const CountParams p)
{
    __shared__ uint32_t s_count[kCountSlice];
    const int b = blockIdx.y, x0 = blockIdx.x * kCountSlice;
    const bool fresh = p.fresh && p.fresh[b] != 0;
    if (p.lens[b] <= 0 && !fresh) return;
    for (int i = threadIdx.x; i < kCountSlice; i += kCountThreads) s_count[i] = 0;
    __syncthreads();
    int len = p.lens[b];
    len = len < p.n ? len : p.n;
    const int prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
    const int32_t *tokens = p.tokens + (int64_t)b * p.n, *path = p.path ? p.path + (int64_t)b * p.n : nullptr;
    const uint32_t end = (uint32_t)(x0 >= p.V ? 0 : p.V - x0 < kCountSlice ? p.V - x0 : kCountSlice);     // (a row may be longer than the vocabulary)
    auto note = [&](int i, int x) {
        const uint32_t at = (uint32_t)(x - x0);                      // (tokens outside the slice, negative ones too, are large)
        if (at >= end) return;
        if (i < prompt) atomicOr(&s_count[at], 0x80000000u);
        else atomicAdd(&s_count[at], 1u);                            // (fewer than 2^31 of them)
    };
    if (path) {
        for (int i = threadIdx.x; i < len; i += kCountThreads) {
            const int at = path[i];
            if (at >= 0 && at < p.n) note(i, tokens[at]);
        }
    } else {
        constexpr int kAhead = 4, kPass = kCountThreads * 4;
        int i = threadIdx.x * 4;
        for (; i + (kAhead - 1) * kPass + 4 <= len; i += kAhead * kPass) {
            i32x4 x[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) __builtin_memcpy(&x[a], tokens + i + a * kPass, 16);      // (rows of odd lengths are aligned to their elements only)
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
#pragma unroll
                for (int k = 0; k < 4; ++k) note(i + a * kPass + k, x[a][k]);
        }
        for (; i < len; i += kPass) {
            if (i + 4 <= len) {
                i32x4 x;
                __builtin_memcpy(&x, tokens + i, 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) note(i + k, x[k]);
            } else {
                for (int k = i; k < len; ++k) note(k, tokens[k]);
            }
        }
    }
    __syncthreads();
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

// A workgroup a row where there are many rows or they are short (up to 12,288 tokens, a row a 256 tokens, 256 rows), else slices: 2,048 workgroups in all as far as
// there are 2,048 tokens for each, and two launches. With everything, us, row and slices: 8,000 tokens, 1 row 9 and 12, 512 rows 17 and 25; 32,003,
// 1 row 17 and 12, 64 rows 21 and 16, 128 rows 23 and 23; 131,072, 1 row 39 and 12, 128 rows 49 and 41, 256 rows 62 and 65, 512 rows 91 and 96.
void probs_plan(ProbsParams &p)
{
    const int64_t rows = (int64_t)p.B * p.n;
    int64_t slices = rows >= 256 || rows * 256 >= p.V || p.V <= 12288 ? 1 : (2048 + rows - 1) / rows;
    const int64_t most = ((int64_t)p.V + kStep - 1) / kStep, least = ((int64_t)p.V + kMostSlice - 1) / kMostSlice;
    if (slices > most) slices = most;
    if (slices < least) slices = least;
    p.slice_len = (int)(((p.V + slices - 1) / slices + kStep - 1) / kStep * kStep);
    p.slices = (int)(((int64_t)p.V + p.slice_len - 1) / p.slice_len);
    p.words = (int)(((int64_t)p.V + 31) / 32);
}

template <typename E, int KIND, bool NT>
static hipError_t launch_probs_t(const ProbsParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)p.B * p.n * p.slices));
    const size_t lds = p.masks || p.n_bias || p.allowed ? (size_t)(p.slice_len < p.V ? p.slice_len : p.V + 31) / 32 * 4 : 0;
    if (p.slices == 1) {
        // Threads of a row, us with 256, 512 and 1,024 of them: 2,048 rows of 700 tokens 15, 26, 45, of 8,000 32, 40, 56; 1,024 rows of 8,000 24, 24, 36, of 16,000 35, 33, 48;
        // 256 rows of 8,000 15, 13, 13; 512 rows of 32,003 38, 31, 32; 256 rows of 131,072 101, 66, 62, 1,024 rows, logits from memory, 235, 229, 212.
        // (65,535 trees of 64 rows of 1,024 threads are as many as a launch takes)
        static_assert(65535LL * kTreeNodes * 1024 <= 0xffffffffLL);
        const int threads = p.V > 65536 ? 1024 : grid.x >= 768 && p.V <= 8192 ? 256 : 512;
        if (threads == 1024) hipLaunchKernelGGL((token_row_kernel<E, 1024, KIND, NT>), grid, dim3(1024), lds, stream, p);
        else if (threads == 512) hipLaunchKernelGGL((token_row_kernel<E, 512, KIND, NT>), grid, dim3(512), lds, stream, p);
        else hipLaunchKernelGGL((token_row_kernel<E, 256, KIND, NT>), grid, dim3(256), lds, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((token_stats_kernel<E, KIND>), grid, dim3(kThreads), lds, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((token_probs_kernel<E, KIND, NT>), grid, dim3(kThreads), lds, stream, p);
    return hipGetLastError();
}

template <typename E, int KIND>
static hipError_t launch_probs_p(const ProbsParams &p, hipStream_t stream)
{
    // Results that no cache holds are stored past the caches, which keep the logits for their second reading (1,024 rows of 131,072 logits, us: bf16 197 -> 169, with a record
    // 227 -> 213; fp32 287 -> 251 and 305 -> 276)
    return (int64_t)p.B * p.n * p.V * 4 >= 128 << 20 ? launch_probs_t<E, KIND, true>(p, stream) : launch_probs_t<E, KIND, false>(p, stream);
}

template <typename E>
static hipError_t launch_probs_e(const ProbsParams &p, hipStream_t stream)
{
    if (p.seen) return launch_probs_p<E, kRecord>(p, stream);
    return p.masks || p.n_bias || p.allowed ? launch_probs_p<E, kNoRecord>(p, stream) : launch_probs_p<E, kPlain>(p, stream);
}

hipError_t launch_token_probs(const ProbsParams &p, int elem_bytes, hipStream_t stream)
{
    return elem_bytes == 2 ? launch_probs_e<uint16_t>(p, stream) : launch_probs_e<float>(p, stream);
}

// Entries by slices from here on, where the row is no longer than a million. 16 requests, 131,072 tokens, us, an entry a thread and slices: 256 entries 2.5 and 3.1 where they are
// spread evenly, 4.4 and 3.1 where half are one of 8,192 tokens, 9.0 and 3.0 where one in 20 is the same; 512 of them 2.8 and 3.2, 7.0 and 3.1, 16.4 and 3.1; 2,048 3.6 and 3.4 and, of
// few tokens, 21 and 3.3. So it is the few entries of a frequent token, which texts have, that decide; evenly spread ones lose half a microsecond up to 1,000. 64 entries: 2.5 and 3.8. A
// million tokens, 512 entries 3 to 13 and 8; four million 3 to 13 and 21.
constexpr int kManyTokens = 256;

hipError_t launch_count_tokens(const CountParams &p, hipStream_t stream)
{
    const int64_t slices = (p.seen_row + kCountSlice - 1) / kCountSlice;
    if (p.n >= kManyTokens && slices <= 128) {
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
