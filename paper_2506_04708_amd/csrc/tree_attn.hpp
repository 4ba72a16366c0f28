// tree_attn.hpp -- attention of the nodes of a drafted tree over a paged key/value cache and over their own ancestors.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace stand {

struct TreeAttnArgs {
    const uint16_t *q, *k_new, *v_new, *k_pool, *v_pool;
    uint16_t *out;
    const int32_t *len, *table, *draft_tok;
    const unsigned long long *anc;
    long long qs[3], ks[3], vs[3], os[3];            // batch, node, head strides in elements
    long long pool_page, pool_slot, pool_head;
    float scale;
    int anc_words, B, N, q_heads, kv_heads, width, pages, page_shift, f16;
};

__device__ __forceinline__ float half_value(uint16_t h, int f16)
{
    return f16 ? (float)__builtin_bit_cast(_Float16, h) : __uint_as_float((uint32_t)h << 16);
}
__device__ __forceinline__ uint16_t half_bits(float f, int f16)
{
    return f16 ? __builtin_bit_cast(uint16_t, (_Float16)f) : __builtin_bit_cast(uint16_t, (__bf16)f);
}

// One workgroup per (trajectory, node, head); its four waves take every fourth key, a lane holds D / 64 elements.
template <int D>
__global__ __launch_bounds__(256) void tree_attn_kernel(TreeAttnArgs a)
{
    constexpr int E = D / 64;
    __shared__ float part[4][D + 2];
    const int b = blockIdx.z, u = blockIdx.y, hq = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int hk = hq / (a.q_heads / a.kv_heads);
    uint16_t *o = a.out + b * a.os[0] + u * a.os[1] + hq * a.os[2] + lane * E;
    if (a.draft_tok[(long long)b * a.N + u] < 0) {
        if (wave == 0)
            for (int e = 0; e < E; ++e) o[e] = 0;
        return;
    }
    const uint16_t *qp = a.q + b * a.qs[0] + u * a.qs[1] + hq * a.qs[2] + lane * E;
    float q[E], acc[E], m = -__builtin_huge_valf(), l = 0.0f;
    for (int e = 0; e < E; ++e) { q[e] = half_value(qp[e], a.f16) * a.scale; acc[e] = 0.0f; }
    long long n = a.len[b];
    const long long most = (long long)a.width << a.page_shift;
    n = n < 0 ? 0 : (n > most ? most : n);
    auto key = [&](const uint16_t *kp, const uint16_t *vp) {
        float s = 0.0f;
        for (int e = 0; e < E; ++e) s += q[e] * half_value(kp[lane * E + e], a.f16);
        for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
        const float m2 = fmaxf(m, s), f = __expf(m - m2), p = __expf(s - m2);
        l = l * f + p;
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + p * half_value(vp[lane * E + e], a.f16);
        m = m2;
    };
    for (long long t = wave; t < n; t += 4) {
        int pg = a.table[(long long)b * a.width + (t >> a.page_shift)];
        pg = pg < 0 ? 0 : (pg >= a.pages ? a.pages - 1 : pg);
        const long long at = pg * a.pool_page + (t & ((1ll << a.page_shift) - 1)) * a.pool_slot + hk * a.pool_head;
        key(a.k_pool + at, a.v_pool + at);
    }
    if (wave == 0)
        for (int v = 0; v <= u; ++v)
            if ((a.anc[(long long)u * a.anc_words + (v >> 6)] >> (v & 63)) & 1ull)
                key(a.k_new + b * a.ks[0] + v * a.ks[1] + hk * a.ks[2], a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2]);
    for (int e = 0; e < E; ++e) part[wave][lane * E + e] = acc[e];
    if (lane == 0) { part[wave][D] = m; part[wave][D + 1] = l; }
    __syncthreads();
    if (wave) return;
    float top = -__builtin_huge_valf(), sum = 0.0f;
    for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w][D]);
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    for (int w = 0; w < 4; ++w) {
        const float f = part[w][D + 1] > 0.0f ? __expf(part[w][D] - top) : 0.0f;
        sum += f * part[w][D + 1];
        for (int e = 0; e < E; ++e) acc[e] += f * part[w][lane * E + e];
    }
    for (int e = 0; e < E; ++e) o[e] = half_bits(acc[e] / sum, a.f16);
}

}  // namespace stand
