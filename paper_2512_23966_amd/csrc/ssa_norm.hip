// Norms of heads with their rotary positions in one pass (gfx950): forward, gradient, and the form of a serving step, whose rows go
// into the cache that decode and extend read.
//
// r = (mean of x_c^2 + eps)^(-1/2) over a head's norm columns; there y_c = x_c r w_c, elsewhere y_c = x_c; then the rotary columns of y
// are rotated (ssa_rope.hip). Gradient: g = the rotation of dout by the negative angle, h = g w on the norm columns,
//     dx_c = r (h_c - x_c r^2 mean(h x)) there, g_c elsewhere,     dw_c = the sum over tokens and heads of g_c x_c r,
// r formed again from x, which is read anyway. All of it in fp32, one rounding of each result.
//
// What bounds it: memory, once there are a few thousand heads: 16,384 tokens of 32 heads of 128 columns 53 us, 5.1 TB/s, and back 70 + 5 (a 1 GiB copy runs at 5.1), in fp32 106,
// 5.1 TB/s, and 157 with the launch that adds; 8,192 tokens of the wide shape into the cache 36 us, 4.2 TB/s (128-byte pieces of rows of 1,152), in fp32 68, 4.5 TB/s; 64 tokens of
// 40 heads 5 us, all latency. A head
// belongs to a group of 8 to 64 lanes of one wave (4 for the narrowest), each with two units of 16 bytes: of rotary columns in half layout
// the two ends of the same pairs, of others any two. So sums are a few exchanges between lanes, a pair is in one lane, and since a lane has the
// same columns of every head it takes, weights and their gradients stay in registers. Rows of 72 units (576 columns) leave 28 of 64 lanes
// idle: 16,384 of them, one a token, 15 us, 2.5 TB/s, and back 24 (fp32, two items a lane: 17, 4.5 TB/s, and 29). A workgroup has one chunk of 8 of them there: its angles, 32 in 64 bits
// a token, wait for its positions, and a group has two rows in all.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_rope.h"
#include "ssa_step.h"

namespace loza {

namespace {

// The columns of a head as items of two units of VEC columns. PAIRS: the items of the rotary columns come first, each with the first
// and the second members of VEC pairs; the other columns follow. Else (interleaved pairs, inside a unit): any two units.
template <int VEC, bool PAIRS>
struct Columns {
    int d, rot, rot_begin;
    bool inter;
    __host__ __device__ int rotary() const { return PAIRS ? rot / 2 / VEC : 0; }
    __host__ __device__ int units() const { return (PAIRS ? d - rot : d) / VEC; }             // of the items behind those
    __host__ __device__ int items() const { return rotary() + (units() + 1) / 2; }
    // first column of unit 0 or 1 of an item; -1: none
    __device__ __forceinline__ int at(int item, int unit) const
    {
        if (PAIRS && item < rotary()) return inter ? rot_begin + 2 * item + unit : rot_begin + item * VEC + unit * (rot / 2);
        const int half = (units() + 1) / 2, u = item - rotary() + unit * half;
        if (item - rotary() >= half || u >= units()) return -1;
        const int c = u * VEC;
        return PAIRS && c >= rot_begin ? c + rot : c;
    }
};

// Sum over the lanes of a group, in all of them (a power of two of lanes, the same in the whole workgroup)
__device__ __forceinline__ float group_sum(float x, int lanes)
{
    if (lanes > 32) x += __shfl_xor(x, 32, 64);
    if (lanes > 16) x += __shfl_xor(x, 16, 64);
    if (lanes > 8) x += __shfl_xor(x, 8, 64);
    if (lanes > 4) x += __shfl_xor(x, 4, 64);
    x += __shfl_xor(x, 2, 64);
    return x + __shfl_xor(x, 1, 64);
}

// What a lane has of every head it takes
template <int VEC, bool PAIRS, int NI>
struct Lane {
    int item[NI], c[NI][2];
    bool normed[NI][2];
    float w[NI][2][VEC];

    __device__ __forceinline__ Lane(const NormHeads &n, int rot, bool inter, int lane, int lanes)
    {
        const Columns<VEC, PAIRS> cols{n.r.d, rot, n.r.rot_begin, inter};
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            item[j] = lane + j * lanes;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                c[j][u] = cols.at(item[j], u);
                normed[j][u] = c[j][u] >= n.norm_begin && c[j][u] < n.norm_begin + n.norm_dim;
#pragma unroll
                for (int e = 0; e < VEC; ++e) w[j][u][e] = normed[j][u] && n.w ? n.w[c[j][u] - n.norm_begin + e] : 1.f;
            }
        }
    }
    template <typename E>
    __device__ __forceinline__ void load(const E *x, Pack<E, VEC> (&raw)[NI][2]) const
    {
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                raw[j][u] = {};
                if (c[j][u] >= 0) raw[j][u] = *(const Pack<E, VEC> *)(x + c[j][u]);
            }
    }
    template <typename E>
    __device__ __forceinline__ static void widen(const Pack<E, VEC> (&raw)[NI][2], float (&v)[NI][2][VEC])
    {
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[j][u][e] = Elem<E>::get(raw[j][u].e[e]);
    }
    template <bool NT, typename E>
    __device__ __forceinline__ void keep(E *out, const float (&v)[NI][2][VEC]) const
    {
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                Pack<E, VEC> p;
#pragma unroll
                for (int e = 0; e < VEC; ++e) p.e[e] = Elem<E>::put(v[j][u][e]);
                if (c[j][u] >= 0) store<NT>(out + c[j][u], p);
            }
    }
    // Rotates by the angles whose (cos, sin) are in sc; sign -1: by the negative ones. (Fused as the compiler fuses them in ssa_rope.hip: the same bits.)
    __device__ __forceinline__ void rotate(float (&v)[NI][2][VEC], const float2 *sc, int rot, int rot_begin, float sign) const
    {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            if constexpr (PAIRS) {
                if (item[j] >= rot / 2 / VEC) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 t = sc[item[j] * VEC + e];
                    const float a = v[j][0][e], b = v[j][1][e], s = sign * t.y;
                    v[j][0][e] = __builtin_fmaf(a, t.x, -(b * s));
                    v[j][1][e] = __builtin_fmaf(b, t.x, a * s);
                }
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (c[j][u] < rot_begin || c[j][u] >= rot_begin + rot) continue;
                    const float2 *at = sc + (c[j][u] - rot_begin) / 2;
#pragma unroll
                    for (int e = 0; e < VEC / 2; ++e) {
                        const float2 t = at[e];
                        const float a = v[j][u][2 * e], b = v[j][u][2 * e + 1], s = sign * t.y;
                        v[j][u][2 * e] = __builtin_fmaf(a, t.x, -(b * s));
                        v[j][u][2 * e + 1] = __builtin_fmaf(b, t.x, a * s);
                    }
                }
            }
        }
    }
    // Sum over the norm columns of the product of a and b
    __device__ __forceinline__ float dot(const float (&a)[NI][2][VEC], const float (&b)[NI][2][VEC], int lanes) const
    {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) part += a[j][u][e] * b[j][u][e];
                sum += normed[j][u] ? part : 0.f;
            }
        return group_sum(sum, lanes);
    }
};

// (cos, sin) of the pairs of the tokens from t0 on, by the whole workgroup
__device__ __forceinline__ void form_angles(const NormParams &p, float2 *sc, int64_t t0, int here)
{
    const int half = p.rot / 2;
    for (int i = threadIdx.x; i < here * half; i += 256) {
        const int t = i / half;
        sc[i] = turn(p.positions[t0 + t], p.freq[i - t * half], p.mscale, false);
    }
}

// The heads that a group of lanes takes: of each chunk of `tokens` tokens that its workgroup takes (every `step`-th) the heads g, g + groups, .. of all of them
struct Rows {
    int64_t T, step, t0;          // t0: first token of the chunk (T and beyond: none is left)
    int tokens, H, groups, g, t, h;

    __device__ __forceinline__ Rows(int64_t T_, int64_t first, int64_t step_, int tokens_, int H_, int groups_, int g_)
        : T(T_), step(step_), t0(first), tokens(tokens_), H(H_), groups(groups_), g(g_), t(0), h(g_)
    {
        settle();
    }
    __device__ __forceinline__ void settle()
    {
        for (; h >= H; h -= H) ++t;
        if (t >= tokens || t0 + t >= T) t0 = T;                      // (a group that finds none in a chunk finds none in later ones)
    }
    __device__ __forceinline__ bool any() const { return t0 < T; }
    __device__ __forceinline__ int64_t token() const { return t0 + t; }
    __device__ __forceinline__ void next()
    {
        h += groups;
        for (; h >= H; h -= H) ++t;
        if (t >= tokens || t0 + t >= T) {
            t0 += step;
            t = 0;
            h = g;
            settle();
        }
    }
};

// Workgroups below q_groups take the queries, those from there on keys (and values). A group asks for its next head before it works on the one it has: the angles of
// a chunk, two tables in turn, are formed while heads are on their way (16,384 tokens of 32 heads 71 -> 53 us, with chunks of 4 tokens in the place of one).
template <typename E, int VEC, bool PAIRS, int NI, bool NT>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormParams p, const int tokens, const int q_groups)
{
    extern __shared__ __attribute__((aligned(16))) float2 sc[];      // [2][tokens][rot / 2]
    const bool keys = (int)blockIdx.x >= q_groups;
    const NormHeads &n = keys ? p.k : p.q;
    const int lanes = n.lanes, half = p.rot / 2;
    const int64_t first = (int64_t)(blockIdx.x - (keys ? q_groups : 0)) * tokens, step = (int64_t)(keys ? gridDim.x - q_groups : q_groups) * tokens;
    const Lane<VEC, PAIRS, NI> lane(n, p.rot, p.interleaved, threadIdx.x & (lanes - 1), lanes);
    Rows rows(p.T, first, step, tokens, n.r.H, 256 / lanes, threadIdx.x / lanes);
    Pack<E, VEC> raw[NI][2];
    int position = -1;
    auto ask = [&]() {
        if (!rows.any()) return;
        lane.load((const E *)n.r.x + rows.token() * n.r.x_token + rows.h * n.r.x_head, raw);
        position = p.positions[rows.token()];
    };
    ask();
    int turn = 0;
    for (int64_t t0 = first; t0 < p.T; t0 += step, turn ^= 1) {
        const int here = (int)(p.T - t0 < tokens ? p.T - t0 : tokens);
        float2 *table = sc + turn * tokens * half;
        form_angles(p, table, t0, here);
        __syncthreads();
        while (rows.t0 == t0) {
            float v[NI][2][VEC];
            lane.widen(raw, v);
            const int64_t tok = rows.token();
            const int t = rows.t, h = rows.h;
            const bool there = position >= 0;
            rows.next();
            ask();
            if (!there) continue;                                    // padding: nothing is written
            int64_t to = tok;
            if (keys) {
                to = p.slots[tok];
                if (to < 0 || to >= p.cache_rows) continue;
            }
            if (n.norm_dim > 0) {
                const float r = 1.f / sqrtf(lane.dot(v, v, lanes) / (float)n.norm_dim + p.eps);
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            if (lane.normed[j][u]) v[j][u][e] = v[j][u][e] * r * lane.w[j][u][e];
            }
            lane.rotate(v, table + t * half, p.rot, n.r.rot_begin, 1.f);
            lane.template keep<NT>((E *)n.r.out + to * n.r.out_token + h * n.r.out_head, v);
        }
        if (!keys || p.v == nullptr) continue;
        using P = Pack<E, VEC>;
        const int per = p.d_v / VEC;
        for (int i = 0; i < here; ++i) {
            const int64_t tok = t0 + i, slot = p.slots[tok];
            if (p.positions[tok] < 0 || slot < 0 || slot >= p.cache_rows) continue;
            for (int k = threadIdx.x; k < per * n.r.H; k += 256) {
                const int vh = k / per, c = (k - vh * per) * VEC;
                *(P *)((E *)p.v_rows + (slot * n.r.H + vh) * p.d_v + c) = *(const P *)((const E *)p.v + tok * p.v_token + vh * p.v_head + c);
            }
        }
    }
}

// Each workgroup leaves one partial sum of dw a column. Three workgroups fit a compute unit (139 registers a lane), and so many are launched: with a third more, 98 us
// in the place of 87 for 16,384 tokens of 32 heads; registers cut to four workgroups are spilled (fp32: 46 -> 82 us).
template <typename E, int VEC, bool PAIRS, int NI, bool NT>
__global__ __launch_bounds__(256) void norm_rope_backward_kernel(const NormParams p, const int tokens)
{
    extern __shared__ __attribute__((aligned(16))) float2 sc[];      // [2][tokens][rot / 2]
    __shared__ float s_dw[256 * NI * 2 * VEC];
    const NormHeads &n = p.q;
    const int lanes = n.lanes, groups = 256 / lanes, half = p.rot / 2;
    const int64_t first = (int64_t)blockIdx.x * tokens, step = (int64_t)gridDim.x * tokens;
    const Lane<VEC, PAIRS, NI> lane(n, p.rot, p.interleaved, threadIdx.x & (lanes - 1), lanes);
    float dw[NI][2][VEC] = {};
    Rows rows(p.T, first, step, tokens, n.r.H, groups, threadIdx.x / lanes);
    Pack<E, VEC> raw_g[NI][2], raw_x[NI][2];
    int position = -1;
    auto ask = [&]() {
        if (!rows.any()) return;
        lane.load((const E *)p.dout + rows.token() * p.dout_token + rows.h * p.dout_head, raw_g);
        lane.load((const E *)n.r.x + rows.token() * n.r.x_token + rows.h * n.r.x_head, raw_x);
        position = p.positions[rows.token()];
    };
    ask();
    int turn = 0;
    for (int64_t t0 = first; t0 < p.T; t0 += step, turn ^= 1) {
        const int here = (int)(p.T - t0 < tokens ? p.T - t0 : tokens);
        float2 *table = sc + turn * tokens * half;
        form_angles(p, table, t0, here);
        __syncthreads();
        while (rows.t0 == t0) {
            float x[NI][2][VEC], g[NI][2][VEC], hw[NI][2][VEC];
            lane.widen(raw_x, x);
            lane.widen(raw_g, g);
            const int64_t tok = rows.token();
            const int t = rows.t, h = rows.h;
            const bool there = position >= 0;
            rows.next();
            ask();
            if (!there) continue;
            lane.rotate(g, table + t * half, p.rot, n.r.rot_begin, -1.f);
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) hw[j][u][e] = g[j][u][e] * lane.w[j][u][e];
            const float inv = 1.f / (float)n.norm_dim;
            const float r = 1.f / sqrtf(lane.dot(x, x, lanes) * inv + p.eps);
            // (r is 0 where the squares add up to infinity: the result is 0 all around, whatever h x adds up to)
            const float hx = lane.dot(hw, x, lanes), mean = r > 0.f ? hx * inv * (r * r) : 0.f;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (lane.normed[j][u]) {
                            dw[j][u][e] += g[j][u][e] * (x[j][u][e] * r);
                            g[j][u][e] = r * (hw[j][u][e] - x[j][u][e] * mean);
                        }
            lane.template keep<NT>((E *)n.r.out + tok * n.r.out_token + h * n.r.out_head, g);
        }
    }
    if (p.partial == nullptr) return;
    // the groups' sums, added in the order of the groups
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s_dw[((j * 2 + u) * VEC + e) * 256 + threadIdx.x] = dw[j][u][e];
    __syncthreads();
    const Columns<VEC, PAIRS> cols{n.r.d, p.rot, n.r.rot_begin, p.interleaved};
    for (int k = threadIdx.x; k < lanes * NI * 2 * VEC; k += 256) {
        const int l = k & (lanes - 1), jue = k / lanes, e = jue % VEC, u = jue / VEC % 2, j = jue / VEC / 2;
        const int c = cols.at(l + j * lanes, u), at = c + e - n.norm_begin;
        if (c < 0 || at < 0 || at >= n.norm_dim) continue;
        float sum = 0.f;
        for (int i = 0; i < groups; ++i) sum += s_dw[jue * 256 + i * lanes + l];
        p.partial[(int64_t)blockIdx.x * n.norm_dim + at] = sum;
    }
}

// dw of 16 columns: 64 rows of threads add every 64th partial sum each, in 64 bits, and then these in a fixed order.
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float *__restrict__ partial, float *__restrict__ dw, int n, int norm_dim)
{
    __shared__ double s_sum[16][16];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), wave = threadIdx.x >> 6;
    double sum = 0;
    if (c < norm_dim) {
#pragma unroll 12
        for (int i = threadIdx.x >> 4; i < n; i += 64) sum += (double)partial[(int64_t)i * norm_dim + c];
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if ((threadIdx.x & 63) < 16) s_sum[wave][threadIdx.x & 15] = sum;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= norm_dim) return;
    sum = 0;
    for (int i = 0; i < 16; ++i) sum += s_sum[i][threadIdx.x];
    dw[c] = (float)sum;
}

constexpr int kNormGroups = 2048;      // workgroups of queries, and of keys, at most

// Lanes of a group: a power of two, at least 4; more than 64 items take several a lane.
template <int VEC, bool PAIRS>
int lanes_of(const NormHeads &n, int rot, bool inter)
{
    const int items = Columns<VEC, PAIRS>{n.r.d, rot, n.r.rot_begin, inter}.items();
    int lanes = 4;
    while (lanes < items && lanes < 64) lanes *= 2;
    return lanes;
}

template <typename E, int VEC, bool PAIRS>
hipError_t launch_t(NormParams p, hipStream_t stream)
{
    constexpr int NI = VEC == 8 ? 1 : VEC == 4 ? 2 : 8;              // 1,024 columns are 64, 128 and 512 items
    p.q.lanes = p.q.r.H ? lanes_of<VEC, PAIRS>(p.q, p.rot, p.interleaved) : 64;
    p.k.lanes = p.k.r.H ? lanes_of<VEC, PAIRS>(p.k, p.rot, p.interleaved) : 64;
    // Tokens of a chunk: as many as give each group of lanes a head, and each thread an angle, where that leaves a thousand chunks
    auto fill = [](const NormHeads &n) { return n.r.H ? (256 / n.lanes + n.r.H - 1) / n.r.H : 1; };
    const int half = p.rot / 2, heads = fill(p.q) > fill(p.k) ? fill(p.q) : fill(p.k), angles = half < 16 ? 16 : (256 + half - 1) / half;
    int tokens = p.T <= 1024 ? 1 : heads;
    if (tokens < angles && p.T / 1024 > tokens) tokens = p.T / 1024 < angles ? (int)(p.T / 1024) : angles;
    const size_t lds = (size_t)2 * tokens * half * sizeof(float2);
    // From 16 MB on results are stored past the caches, which keep x for the gradient: forward and gradient, 16 MB 27 -> 24 us, 32 MB 41 -> 38, 64 MB 67 and 67, 128 MB
    // 132 -> 122, 256 MB 264 -> 255. (What reads the forward's result next, an addition: 16 and 32 MB 22 -> 20 and 28 -> 28 us, 128 MB 86 -> 95, 256 MB 195 -> 199.)
    const bool past = VEC > 1 && p.k.r.H == 0 && p.T > ((16 << 20) - 1) / ((int64_t)p.q.r.H * p.q.r.d * (int64_t)sizeof(E));
    const int64_t blocks = (p.T + tokens - 1) / tokens;
    if (p.dout) {
        const int n = (int)(blocks < kNormPartials ? blocks : kNormPartials);
        float *dw = p.dw;
        if (n == 1 && dw) p.partial = dw;                            // (one workgroup's sums are the sums)
        if (past) hipLaunchKernelGGL((norm_rope_backward_kernel<E, VEC, PAIRS, NI, true>), dim3((unsigned)n), dim3(256), lds, stream, p, tokens);
        else hipLaunchKernelGGL((norm_rope_backward_kernel<E, VEC, PAIRS, NI, false>), dim3((unsigned)n), dim3(256), lds, stream, p, tokens);
        if (dw == nullptr || n == 1) return hipGetLastError();
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        hipLaunchKernelGGL(norm_dw_kernel, dim3((unsigned)((p.q.norm_dim + 15) / 16)), dim3(1024), 0, stream, (const float *)p.partial, dw, n, p.q.norm_dim);
        return hipGetLastError();
    }
    const int most = (int)(blocks < kNormGroups ? blocks : kNormGroups), q_groups = p.q.r.H ? most : 0;
    const dim3 grid((unsigned)(q_groups + (p.k.r.H ? most : 0)));
    if (past) hipLaunchKernelGGL((norm_rope_kernel<E, VEC, PAIRS, NI, true>), grid, dim3(256), lds, stream, p, tokens, q_groups);
    else hipLaunchKernelGGL((norm_rope_kernel<E, VEC, PAIRS, NI, false>), grid, dim3(256), lds, stream, p, tokens, q_groups);
    return hipGetLastError();
}

template <typename E, int VEC>
hipError_t launch_v(const NormParams &p, hipStream_t stream)
{
    if constexpr (VEC > 1) {
        if (p.interleaved) return launch_t<E, VEC, false>(p, stream);
    }
    return launch_t<E, VEC, true>(p, stream);
}

}  // namespace

hipError_t launch_norm_rope(const NormParams &p, int elem_bytes, hipStream_t stream)
{
    const int vec = 16 / elem_bytes;
    auto whole = [&](int64_t x) { return x % vec == 0; };
    auto at16 = [](const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
    auto heads = [&](const NormHeads &n) {
        return n.r.H == 0 || (at16(n.r.x) && at16(n.r.out) && whole(n.r.x_token) && whole(n.r.x_head) && whole(n.r.out_token) && whole(n.r.out_head) &&
                              whole(n.r.d) && whole(n.r.rot_begin) && whole(n.norm_begin) && whole(n.norm_dim));
    };
    const bool wide = heads(p.q) && heads(p.k) && whole(p.interleaved ? p.rot : p.rot / 2) &&
                      (p.v == nullptr || (at16(p.v) && at16(p.v_rows) && whole(p.v_token) && whole(p.v_head) && whole(p.d_v))) &&
                      (p.dout == nullptr || (at16(p.dout) && whole(p.dout_token) && whole(p.dout_head)));
    if (elem_bytes == 2) return wide ? launch_v<uint16_t, 8>(p, stream) : launch_v<uint16_t, 1>(p, stream);
    return wide ? launch_v<float, 4>(p, stream) : launch_v<float, 1>(p, stream);
}

}  // namespace loza
