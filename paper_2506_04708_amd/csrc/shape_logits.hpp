// shape_logits.hpp -- penalties for repeated tokens, biases and grammar masks on the logits of every node of a drafted tree.
//
// For trajectory b, drafted node u and token v: c = times v was generated, plus its occurrences on the path root -> u (the
// root itself has been counted), seen = c > 0 or v occurs in the prompt, and in this order
//     x <- seen ? (x > 0 ? x / repetition : x * repetition) : x
//     x <- x - frequency * c
//     x <- x - presence            where c > 0
//     x <- x + bias[v]
//     x <- -inf                    where the row's mask has no bit for v, unless it has no bit at all
// in binary32, rounded once to the type of the logits.
#pragma once
#include "wave_ops.hpp"

namespace stand {

constexpr int kPromptFlag = 1 << 30;   // count[b][v]: bits 0 .. 29 times generated, bit 30: occurs in the prompt
constexpr int kShapeThreads = 256;
constexpr int kShapeTokens = 8;        // consecutive tokens of a thread
constexpr int kShapeSpan = kShapeThreads * kShapeTokens;

struct ShapeArgs {
    const void *x;
    void *out;
    const int32_t *draft_tok, *count, *bias_id;
    const float *penalty, *bias;
    const uint32_t *allow;
    const unsigned long long *anc;
    int anc_words, N, V, M, words, nodes_per_group, node_groups;
};

struct alignas(2) Half8 { uint16_t h[8]; };   // eight logits at any alignment: rows of an odd vocabulary start anywhere
struct alignas(4) Float8 { float f[8]; };
struct alignas(4) Int8 { int32_t i[8]; };

template <int DT>
__device__ __forceinline__ void load_tokens(const void *row, int t, float (&x)[8])
{
    if constexpr (DT == kDtBf16) {
        const Half8 w = *(const Half8 *)((const uint16_t *)row + t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = u2f((uint32_t)w.h[i] << 16);
    } else {
        const Float8 w = *(const Float8 *)((const float *)row + t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = w.f[i];
    }
}

// Nearest bf16, ties to even; infinities stay, a NaN stays one.
__device__ __forceinline__ uint16_t bf16_bits(float f)
{
    const uint32_t u = f2u(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);
    return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

template <int DT>
__device__ __forceinline__ void store_tokens(void *row, int t, const float (&x)[8])
{
    if constexpr (DT == kDtBf16) {
        Half8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.h[i] = bf16_bits(x[i]);
        *(Half8 *)((uint16_t *)row + t) = w;
    } else {
        Float8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.f[i] = x[i];
        *(Float8 *)((float *)row + t) = w;
    }
}

template <int DT>
__global__ __launch_bounds__(kShapeThreads) void shape_logits_kernel(ShapeArgs a)
{
    __shared__ int32_t slot[kShapeSpan];          // last entry of the bias list for each token of the span
    __shared__ uint16_t hit_node[kMaxNodes], hit_at[kMaxNodes];
    __shared__ int hits;
    const int b = blockIdx.y, tid = threadIdx.x;
    const int span = blockIdx.x / a.node_groups, group = blockIdx.x % a.node_groups;
    const int t0 = span * kShapeSpan, t = t0 + tid * kShapeTokens;
    const int mine = a.V - t < 0 ? 0 : (a.V - t < 8 ? a.V - t : 8);
    const int32_t *tok = a.draft_tok + (long long)b * a.N;

    if (tid == 0) hits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) slot[tid * 8 + i] = -1;
    __syncthreads();
    for (int u = 1 + tid; u < a.N; u += kShapeThreads) {
        const int at = tok[u] - t0;
        if (tok[u] >= 0 && at >= 0 && at < kShapeSpan) {
            const int q = atomicAdd(&hits, 1);
            hit_node[q] = (uint16_t)u;
            hit_at[q] = (uint16_t)at;
        }
    }
    for (int i = tid; i < a.M; i += kShapeThreads) {
        const int id = a.bias_id[(long long)b * a.M + i];
        if (id >= t0 && id < t0 + kShapeSpan && id < a.V) atomicMax(&slot[id - t0], i);
    }
    __syncthreads();

    int32_t c0[8];
    float shift[8];
    const float rho = a.penalty ? a.penalty[3 * (long long)b] : 1.0f;
    const float present = a.penalty ? a.penalty[3 * (long long)b + 1] : 0.0f;
    const float often = a.penalty ? a.penalty[3 * (long long)b + 2] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c0[i] = a.count && i < mine ? a.count[(long long)b * a.V + t + i] : 0;
        const int s = a.M ? slot[tid * 8 + i] : -1;
        shift[i] = s >= 0 ? a.bias[(long long)b * a.M + s] : 0.0f;
    }
    bool near = false;
    for (int q = 0; q < hits; ++q) near |= hit_at[q] / 8 == tid;

    const int u1 = min(a.N, (group + 1) * a.nodes_per_group);
    for (int u = group * a.nodes_per_group; u < u1; ++u) {
        const long long r = (long long)b * a.N + u;
        const char *xr = (const char *)a.x + r * a.V * VecTraits<DT>::ES;
        char *yr = (char *)a.out + r * a.V * VecTraits<DT>::ES;
        const bool drafted = tok[u] >= 0;
        if (!drafted && a.x == a.out) continue;
        unsigned keep = 0xFFu;
        if (a.allow && drafted) {
            const uint32_t *m = a.allow + r * a.words;
            const unsigned valid = (1u << mine) - 1u;
            keep = mine ? (m[t >> 5] >> (t & 31)) & valid : 0u;
            if (!__syncthreads_or(keep != 0)) {
                // none in this span: -inf everywhere, unless the row has no bit at all
                bool any = false;
                for (int w0 = 0; w0 < a.words && !any; w0 += 4 * kShapeThreads) {
                    uint32_t got = 0;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int w = w0 + q * kShapeThreads + tid;
                        if (w < a.words) got |= m[w] & (w == a.words - 1 && (a.V & 31) ? (1u << (a.V & 31)) - 1u : ~0u);
                    }
                    any = __syncthreads_or(got != 0);
                }
                if (!any) keep = 0xFFu;
            }
        }
        if (!mine) continue;
        float x[8];
        if (mine == 8) load_tokens<DT>(xr, t, x);
        else
            for (int i = 0; i < 8; ++i) x[i] = i < mine ? load_scalar<DT>(xr, t + i) : 0.0f;
        if (drafted) {
            int32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = c0[i];
            if (near)
                for (int q = 0; q < hits; ++q) {
                    const int v = hit_node[q], at = hit_at[q] - tid * 8;
                    const bool on = (a.anc[(long long)u * a.anc_words + (v >> 6)] >> (v & 63)) & 1ull;
#pragma unroll
                    for (int i = 0; i < 8; ++i) c[i] += on && at == i ? 1 : 0;
                }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float times = (float)(c[i] & (kPromptFlag - 1));
                float y = x[i];
                if (c[i] != 0) {
                    y = y > 0.0f ? y / rho : y * rho;
                    y = y - often * times;
                    y = times > 0.0f ? y - present : y;
                }
                y = y + shift[i];
                x[i] = (keep >> i) & 1u ? y : -__builtin_huge_valf();
            }
        }
        if (mine == 8) store_tokens<DT>(yr, t, x);
        else
            for (int i = 0; i < mine; ++i) {
                if constexpr (DT == kDtBf16) ((uint16_t *)yr)[t + i] = bf16_bits(x[i]);
                else ((float *)yr)[t + i] = x[i];
            }
    }
}

// Tokens into the counts: the prompt's set a flag, generated ones are added.
__global__ __launch_bounds__(256) void count_tokens_kernel(int32_t *count, const int32_t *tok, const int32_t *len, int V, int width, int prompt)
{
    const int b = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
    if (j >= width || (len && j >= len[b])) return;
    const int v = tok[(long long)b * width + j];
    if (v < 0 || v >= V) return;
    int32_t *c = count + (long long)b * V + v;
    if (!prompt) atomicAdd(c, 1);
    else if (!(*c & kPromptFlag)) atomicOr(c, kPromptFlag);
}

}  // namespace stand
