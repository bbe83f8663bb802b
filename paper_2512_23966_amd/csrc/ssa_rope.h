// Device code of rotary positions that its kernels share (ssa_rope.hip, ssa_norm.hip): angles, elements, stores.
//
// Angles of far positions need more than 24 bits: position 2^20 times a frequency of 1 leaves 4 bits behind the point in fp32.
// They are formed as turns in two doubles, reduced to an eighth of a turn there, and only then rounded to fp32.
#ifndef LOZA_SSA_ROPE_H
#define LOZA_SSA_ROPE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"

namespace loza {

namespace {

// m cos and m sin of pos * freq (freq in radians per position)
__device__ __forceinline__ float2 turn(int32_t pos, double freq, float m, bool inverse)
{
    // freq / pi and pos * freq / pi as sums of two doubles: the error is below 2^-70 of a half turn per position
    constexpr double kInvPi = 0.31830988618379067154, kInvPiLo = -1.9678676675182486e-17;   // 1 / pi
    const double fh = freq * kInvPi, fl = __builtin_fma(freq, kInvPi, -fh) + freq * kInvPiLo;
    const double i = (double)pos, h = i * fh, l = __builtin_fma(i, fh, -h) + i * fl;
    const double a = (h - 2.0 * __builtin_rint(0.5 * h)) + l;   // half turns, about [-1, 1]
    const double k = __builtin_rint(2.0 * a);                   // the nearest quarter of a turn, and what is left of it
    float s, c;
    sincospif((float)(a - 0.5 * k), &s, &c);
    const int q = (int)k & 3;
    const float si = (q & 1) ? c : s, co = (q & 1) ? s : c;
    const float sine = (q & 2) ? -si : si, cosine = (q == 1 || q == 2) ? -co : co;
    return make_float2(m * cosine, inverse ? -m * sine : m * sine);
}

template <typename E> struct Elem;
template <> struct Elem<uint16_t> {
    static __device__ __forceinline__ float get(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
    static __device__ __forceinline__ uint16_t put(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }   // the one rounding
};
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
};
template <typename E, int N> struct alignas(sizeof(E) * N) Pack { E e[N]; };

// NT: past the caches (16-byte stores only)
template <bool NT, typename P>
__device__ __forceinline__ void store(void *at, const P &v)
{
    if constexpr (NT && sizeof(P) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4 *)at);
    else *(P *)at = v;
}

}  // namespace

}  // namespace loza
#endif
