// Attention of a tree of drafted tokens over a cache (gfx950), in its plainest form: a wave per (node, query head), the lanes
// share a row's columns.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssa_device.h"
#include "ssa_kernels.h"
#include "ssa_tree.h"

namespace loza {

template <int DQK, int DV>
__global__ __launch_bounds__(64) void tree_plain_kernel(const FwdParams p, const bool alias)
{
    constexpr int NQ = DQK / 64, NV = DV / 64;
    const int lane = threadIdx.x;
    int64_t id = blockIdx.x;
    const int h = (int)(id % p.Hq);
    id /= p.Hq;
    const int r = (int)(id % p.q_len), b = (int)(id / p.q_len), g = h / p.G;
    const TreeSpan span = tree_span(p, b);
    const TreeRow row = tree_row(p, span, b, r);
    float q[NQ], o[NV], m = LOZA_NEG_INF, l = 0.f;
    const int64_t q_row = ((int64_t)b * p.q_len + r) * p.Hq + h;
    auto widen = [](uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); };
    for (int e = 0; e < NQ; ++e) q[e] = widen(p.q[q_row * DQK + e * 64 + lane]);
    for (int e = 0; e < NV; ++e) o[e] = 0.f;
    for (int64_t j = 0; j < span.L; ++j) {
        const bool ok = j < span.P ? row.seen && (j < p.n_sink || j >= row.w_lo) : (row.mask >> (j - span.P)) & 1;
        if (!ok) continue;
        int64_t at = (int64_t)b * p.S + j;
        if (p.block_table) {
            int64_t pid = p.block_table[(int64_t)b * p.max_pages + (j >> p.page_shift)];
            pid = pid < 0 ? 0 : pid < p.num_pages ? pid : p.num_pages - 1;
            at = (pid << p.page_shift) + (j & ((1 << p.page_shift) - 1));
        }
        at = at * p.Hkv + g;
        float s = 0.f;
        for (int e = 0; e < NQ; ++e) s += q[e] * widen(p.k[at * DQK + e * 64 + lane]);
        for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
        s *= p.scale_log2;
        const float m_new = fmaxf(m, s), a = exp2f(m - m_new), w = exp2f(s - m_new);
        m = m_new;
        l = l * a + w;
        const uint16_t *v = alias ? p.k + at * DQK : p.v + at * DV;
        for (int e = 0; e < NV; ++e) o[e] = o[e] * a + w * widen(v[e * 64 + lane]);
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    for (int e = 0; e < NV; ++e) p.out[q_row * DV + e * 64 + lane] = __builtin_bit_cast(uint16_t, (__bf16)(o[e] * inv));
    if (lane == 0) p.lse[((int64_t)b * p.Hq + h) * p.q_len + r] = (m + log2f(l)) * 0.69314718055994530942f;
}

hipError_t launch_tree_plain(const FwdParams &p, int d_qk, bool alias, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)p.B * p.q_len * p.Hq));
    if (d_qk == 576) hipLaunchKernelGGL((tree_plain_kernel<576, 512>), grid, dim3(64), 0, stream, p, alias);
    else hipLaunchKernelGGL((tree_plain_kernel<128, 128>), grid, dim3(64), 0, stream, p, alias);
    return hipGetLastError();
}

}  // namespace loza
