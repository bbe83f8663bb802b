// Rotary positions (gfx950): the rotation of query and key heads, its gradient, and the same with the new rows written into
// the cache that decode and extend read.
//
// A pair (a, b) of a head's rotary columns at position i becomes m (a cos - b sin, a sin + b cos), the angle i * freq[pair].
// The gradient of that is the rotation by the negative angle with the same m (`inverse`). Pairs are neighbours (interleaved)
// or columns rot / 2 apart (half layout); columns outside [rot_begin, rot_begin + rot) are copied, or left where the call is in place.
//
// What bounds it: memory. A workgroup takes a few tokens: it forms the sines and cosines of its tokens once, in LDS, for
// all heads (64 heads of the wide shape use each of them 64 times), then moves 16 bytes a lane.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_rope.h"
#include "ssa_step.h"

namespace loza {

namespace {

// The heads of one token, by all threads of the workgroup. VEC elements a load (1: rows or columns that are not aligned to
// 16 bytes); sc: (cos, sin) of the token's pairs.
template <typename E, int VEC, bool INTER, bool NT>
__device__ __forceinline__ void rotate_heads(const RopeHeads &r, const E *x, E *out, int rot, const float2 *sc, bool copy_rest)
{
    using P = Pack<E, VEC>;
    constexpr int PAIRS = INTER ? (VEC > 1 ? VEC / 2 : 1) : VEC;    // pairs a unit rotates
    const int units = rot / 2 / PAIRS, rest = copy_rest ? (r.d - rot) / VEC : 0, per = units + rest, n = per * r.H;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int h = i / per, u = i - h * per;
        const E *xh = x + h * r.x_head;
        E *oh = out + h * r.out_head;
        if (u >= units) {                                            // a column outside the rotary ones
            int c = (u - units) * VEC;
            c = c < r.rot_begin ? c : c + rot;
            store<NT>(oh + c, *(const P *)(xh + c));
            continue;
        }
        if constexpr (INTER && VEC > 1) {
            const int c = r.rot_begin + u * VEC;
            P v = *(const P *)(xh + c);
#pragma unroll
            for (int e = 0; e < PAIRS; ++e) {
                const float2 t = sc[u * PAIRS + e];
                const float a = Elem<E>::get(v.e[2 * e]), b = Elem<E>::get(v.e[2 * e + 1]);
                v.e[2 * e] = Elem<E>::put(a * t.x - b * t.y);
                v.e[2 * e + 1] = Elem<E>::put(a * t.y + b * t.x);
            }
            store<NT>(oh + c, v);
        } else {
            const int c0 = r.rot_begin + (INTER ? 2 * u : u * VEC), c1 = INTER ? c0 + 1 : c0 + rot / 2;
            P v = *(const P *)(xh + c0), w = *(const P *)(xh + c1);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float2 t = sc[u * PAIRS + e];
                const float a = Elem<E>::get(v.e[e]), b = Elem<E>::get(w.e[e]);
                v.e[e] = Elem<E>::put(a * t.x - b * t.y);
                w.e[e] = Elem<E>::put(a * t.y + b * t.x);
            }
            store<NT>(oh + c0, v);
            store<NT>(oh + c1, w);
        }
    }
}

template <typename E, int VEC, bool INTER, bool NT>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams p, const int tokens)
{
    extern __shared__ __attribute__((aligned(16))) float2 sc[];      // [tokens][rot / 2]
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int half = p.rot / 2, here = (int)(p.T - t0 < tokens ? p.T - t0 : tokens);
    for (int i = threadIdx.x; i < here * half; i += 256) {
        const int t = i / half;
        sc[i] = turn(p.positions[t0 + t], p.freq[i - t * half], p.mscale, p.inverse);
    }
    __syncthreads();
    for (int t = 0; t < here; ++t) {
        const int64_t tok = t0 + t;
        if (p.positions[tok] < 0) continue;                          // padding: nothing is written
        const float2 *s = sc + t * half;
        if (p.q.H > 0)
            rotate_heads<E, VEC, INTER, NT>(p.q, (const E *)p.q.x + tok * p.q.x_token, (E *)p.q.out + tok * p.q.out_token, p.rot, s, p.q.x != p.q.out);
        if (p.k.H == 0) continue;
        const int64_t slot = p.slots[tok];
        if (slot < 0 || slot >= p.cache_rows) continue;
        rotate_heads<E, VEC, INTER, false>(p.k, (const E *)p.k.x + tok * p.k.x_token, (E *)p.k.out + slot * p.k.out_token, p.rot, s, true);
        if (p.v == nullptr) continue;
        using P = Pack<E, VEC>;
        const int per = p.d_v / VEC;
        for (int i = threadIdx.x; i < per * p.k.H; i += 256) {
            const int h = i / per, c = (i - h * per) * VEC;
            *(P *)((E *)p.v_rows + (slot * p.k.H + h) * p.d_v + c) = *(const P *)((const E *)p.v + tok * p.v_token + h * p.v_head + c);
        }
    }
}

template <typename E, int VEC, bool INTER>
hipError_t launch_t(const RopeParams &p, hipStream_t stream)
{
    // Two tokens a workgroup (16,384 tokens of 64 heads of 64 columns, and back: one 81.3 us, two 80.8, four 86.8; 8,192 of 32 heads of
    // 128, fp32: 82.9, 87.4, 90.3; into rows of 576: 110, 103, 101), one where there are few. Results that no cache holds, 32 MB and more, are stored
    // past the caches (the same three 81 us in the place of 103, 87 of 130, 103 of 115).
    const int tokens = p.T <= 2048 ? 1 : 2;
    const dim3 grid((unsigned)((p.T + tokens - 1) / tokens));
    const size_t lds = (size_t)tokens * (p.rot / 2) * sizeof(float2);
    const bool past = VEC > 1 && p.k.H == 0 && p.q.x != p.q.out && p.T * p.q.H * p.q.d * (int64_t)sizeof(E) >= 32 << 20;
    if constexpr (VEC > 1) {
        if (past) {
            hipLaunchKernelGGL((rope_kernel<E, VEC, INTER, true>), grid, dim3(256), lds, stream, p, tokens);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((rope_kernel<E, VEC, INTER, false>), grid, dim3(256), lds, stream, p, tokens);
    return hipGetLastError();
}

template <typename E, int VEC>
hipError_t launch_v(const RopeParams &p, hipStream_t stream)
{
    return p.interleaved ? launch_t<E, VEC, true>(p, stream) : launch_t<E, VEC, false>(p, stream);
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, int elem_bytes, hipStream_t stream)
{
    const int vec = 16 / elem_bytes;
    auto whole = [&](int64_t x) { return x % vec == 0; };
    auto at16 = [](const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
    auto heads = [&](const RopeHeads &r) {
        return r.H == 0 || (at16(r.x) && at16(r.out) && whole(r.x_token) && whole(r.x_head) && whole(r.out_token) && whole(r.out_head) && whole(r.d) &&
                            whole(r.rot_begin));
    };
    const bool wide = heads(p.q) && heads(p.k) && whole(p.interleaved ? p.rot : p.rot / 2) &&
                      (p.v == nullptr || (at16(p.v) && at16(p.v_rows) && whole(p.v_token) && whole(p.v_head) && whole(p.d_v)));
    // (a launch has fewer than 2^32 threads in x: 2^23 workgroups at most for these tokens, and calls of more in parts)
    constexpr int64_t kMostTokens = 1 << 24;
    RopeParams part = p;
    for (int64_t t0 = 0; t0 < p.T; t0 += kMostTokens) {
        auto from = [&](const void *x, int64_t token) { return x ? (const char *)x + t0 * token * elem_bytes : nullptr; };
        part.T = p.T - t0 < kMostTokens ? p.T - t0 : kMostTokens;
        part.q.x = from(p.q.x, p.q.x_token);
        part.q.out = (void *)from(p.q.out, p.q.out_token);
        part.k.x = from(p.k.x, p.k.x_token);                          // (rows of the cache are by slot)
        part.v = from(p.v, p.v_token);
        part.positions = p.positions + t0;
        part.slots = p.slots ? p.slots + t0 : nullptr;
        const hipError_t e = elem_bytes == 2 ? (wide ? launch_v<uint16_t, 8>(part, stream) : launch_v<uint16_t, 1>(part, stream))
                                             : (wide ? launch_v<float, 4>(part, stream) : launch_v<float, 1>(part, stream));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace loza
