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
#include "row_words.hpp"
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
    uint8_t *any;                  // workspace: [B][N], 1 where a row's mask has a bit for a token
    const unsigned long long *anc;
    int anc_words, N, V, M, words, nodes_per_group, node_groups, spans;
    long long rows;
};

struct Half8 { uint16_t h[8]; };
struct Float4 { float f[4]; };
struct Int4 { uint32_t i[4]; };        // counts and mask words: aligned like one of them

// (Streamed past the caches: 296 us instead of 308 us for 32 trees of 64 rows of 152064.)
template <int DT>
__device__ __forceinline__ void load_tokens(const void *row, int t, float (&x)[8])
{
    if constexpr (DT == kDtBf16) {
        const Half8 w = __builtin_bit_cast(Half8, __builtin_nontemporal_load((const RowWords<2>::type *)((const uint16_t *)row + t)));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = u2f((uint32_t)w.h[i] << 16);
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const Float4 w = __builtin_bit_cast(Float4, __builtin_nontemporal_load((const RowWords<4>::type *)((const float *)row + t + 4 * q)));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * q + i] = w.f[i];
        }
    }
}

// Nearest bf16, ties to even (one instruction for two of them).
__device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

template <int DT>
__device__ __forceinline__ void store_tokens(void *row, int t, const float (&x)[8])
{
    if constexpr (DT == kDtBf16) {
        Half8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.h[i] = bf16_bits(x[i]);
        __builtin_nontemporal_store(__builtin_bit_cast(RowWords<2>::type, w), (RowWords<2>::type *)((uint16_t *)row + t));
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const Float4 w = {{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]}};
            __builtin_nontemporal_store(__builtin_bit_cast(RowWords<4>::type, w), (RowWords<4>::type *)((float *)row + t + 4 * q));
        }
    }
}

// Which rows' masks have a bit for a token at all: one wave per row, 8 KiB of bits in flight, done at the first bit.  (Made by
// the workgroups of the kernel below for themselves, this cost 83 us, this kernel takes 9.5: they wait where they should stream.)
__global__ __launch_bounds__(256) void shape_rows_kernel(ShapeArgs a)
{
    const int lane = threadIdx.x & 63;
    const long long r = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (r >= a.rows || a.draft_tok[r] < 0) return;
    const uint32_t *m = a.allow + r * a.words;
    bool any = false;
    for (int w0 = 0; w0 < a.words && !any; w0 += 8 * 4 * 64) {
        uint32_t x = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int w = w0 + (q * 64 + lane) * 4;
            if (w + 4 < a.words) {
                const Int4 y = *(const Int4 *)(m + w);
                x |= y.i[0] | y.i[1] | y.i[2] | y.i[3];
            } else {
                for (int e = w; e < a.words; ++e) x |= m[e] & (e == a.words - 1 && (a.V & 31) ? (1u << (a.V & 31)) - 1u : ~0u);
            }
        }
        any = __ballot(x != 0) != 0;
    }
    if (lane == 0) a.any[r] = any;
}

// A workgroup has one span of tokens for up to kShapeNodes nodes of a trajectory: counts and biases of its tokens are read
// once and stay in registers, and so do the mask bits of all its nodes, so that the nodes' rows pass without a barrier between
// them, kShapeAhead at a time.  In fp32 these are in flight together; in bf16 each is unpacked where it is loaded, so a thread has
// one row in flight and the other waves of the compute unit have theirs.  What a mask leaves nothing of is not read.  Bound by
// HBM where there is much to do (2048 rows of 152064: 289 us, 4.5 TB/s): logits in and out, mask bits, counts once for every
// kShapeNodes nodes; else by the chain nodes -> mask, counts and biases -> rows (16 rows of 32000 in fp32: 5.8 us, 64 rows of 50257:
// 11 us).  In place, rows that were not drafted are read all the same.
constexpr int kShapeNodes = 16, kShapeAhead = 4;

template <int DT>
__global__ __launch_bounds__(kShapeThreads) void shape_logits_kernel(ShapeArgs a)
{
    __shared__ int32_t slot[kShapeSpan];          // last entry of the bias list for each token of the span
    __shared__ uint16_t hit_node[kMaxNodes], hit_at[kMaxNodes];
    __shared__ int hits;
    const int tid = threadIdx.x;
    const int group = blockIdx.x % a.node_groups, span = blockIdx.x / a.node_groups % a.spans;
    const long long b = blockIdx.x / a.node_groups / a.spans;
    const int t0 = span * kShapeSpan, t = t0 + tid * kShapeTokens;
    const int mine = a.V - t < 0 ? 0 : (a.V - t < 8 ? a.V - t : 8);
    const int32_t *tok = a.draft_tok + b * a.N;
    const int u0 = group * a.nodes_per_group, nodes = min(a.N - u0, a.nodes_per_group);
    const long long r0 = b * a.N + u0;

    // mask bits of this thread's tokens, a byte for every node; rows that are not masked keep all of them
    uint32_t keep[kShapeNodes / 4] = {~0u, ~0u, ~0u, ~0u};
    int drafted, masked;                          // bit per node
    {
        const int lane = tid & 63;
        const bool here = lane < nodes;
        const int v = here ? tok[u0 + lane] : -1;
        const bool any = a.allow && here && a.any[r0 + lane];
        drafted = (int)__ballot(v >= 0);
        masked = (int)__ballot(any) & drafted;    // (nothing has been written for the other rows)
    }
    if (masked) {
        uint32_t got[kShapeNodes];
#pragma unroll
        for (int i = 0; i < kShapeNodes; ++i) got[i] = (masked >> i & 1) && mine ? a.allow[(r0 + i) * a.words + (t >> 5)] : 0u;
#pragma unroll
        for (int i = 0; i < kShapeNodes; ++i)
            if (masked >> i & 1) keep[i / 4] = (keep[i / 4] & ~(0xFFu << (i % 4 * 8))) | (got[i] >> (t & 31) & 0xFFu) << (i % 4 * 8);
    }

    // the bias of each token (of several entries the last), drafted tokens of the span
    if (tid == 0) hits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) slot[tid * 8 + i] = -1;
    __syncthreads();
    for (int u = 1 + tid; u < a.N; u += kShapeThreads) {
        const int v = tok[u], at = v - t0;
        if (v >= 0 && at >= 0 && at < kShapeSpan) {
            const int q = atomicAdd(&hits, 1);
            hit_node[q] = (uint16_t)u;
            hit_at[q] = (uint16_t)at;
        }
    }
    for (int i = tid; i < a.M; i += kShapeThreads) {
        const int id = a.bias_id[b * a.M + i];
        if (id >= t0 && id < t0 + kShapeSpan && id < a.V) atomicMax(&slot[id - t0], i);
    }
    __syncthreads();

    int32_t c0[8];
    float shift[8];
    const float rho = a.penalty ? a.penalty[3 * b] : 1.0f, inverse = 1.0f / rho;
    const float divisor = rho < __builtin_huge_valf() ? rho : 0.0f;   // (an infinite one's quotients are zero without a remainder)
    const float present = a.penalty ? a.penalty[3 * b + 1] : 0.0f;
    const float often = a.penalty ? a.penalty[3 * b + 2] : 0.0f;
    bool touched = false;                         // this thread's tokens are not all as they were
    if (a.count && mine == 8) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const Int4 w = *(const Int4 *)(a.count + b * a.V + t + 4 * q);
#pragma unroll
            for (int i = 0; i < 4; ++i) c0[4 * q + i] = (int32_t)w.i[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c0[i] = a.count && i < mine ? a.count[b * a.V + t + i] : 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int s = slot[tid * 8 + i];
        shift[i] = s >= 0 ? a.bias[b * a.M + s] : 0.0f;
        touched |= c0[i] != 0 || s >= 0;
    }
    bool near = false;
    for (int q = 0; q < hits; ++q) near |= hit_at[q] / 8 == tid;
    touched |= near;
    if (!mine) return;

    const long long row = (long long)a.V * VecTraits<DT>::ES;
    const char *xp = (const char *)a.x + r0 * row;
    char *yp = (char *)a.out + r0 * row;
    for (int i0 = 0; i0 < nodes; i0 += kShapeAhead) {
        float x[kShapeAhead][8];
        const uint32_t kept = i0 == 0 ? keep[0] : i0 == 4 ? keep[1] : i0 == 8 ? keep[2] : keep[3];
#pragma unroll
        for (int k = 0; k < kShapeAhead; ++k) {
            const int i = i0 + k;
            if (i < nodes && (kept >> (k * 8) & 0xFFu)) {
                if (mine == 8) load_tokens<DT>(xp + i * row, t, x[k]);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[k][e] = e < mine ? load_scalar<DT>(xp + i * row, t + e) : 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < kShapeAhead; ++k) {
            const int i = i0 + k;
            if (i >= nodes || (!(drafted >> i & 1) && a.x == a.out)) continue;
            if (drafted >> i & 1) {
                if (touched) {
                    int32_t c[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) c[e] = c0[e];
                    if (near)
                        for (int q = 0; q < hits; ++q) {
                            const int v = hit_node[q], at = hit_at[q] - tid * 8;
                            const bool on = (a.anc[(long long)(u0 + i) * a.anc_words + (v >> 6)] >> (v & 63)) & 1ull;
#pragma unroll
                            for (int e = 0; e < 8; ++e) c[e] += on && at == e ? 1 : 0;
                        }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float times = (float)(c[e] & (kPromptFlag - 1)), z = x[k][e];
                        // the quotient to half a step: one correction with the exact remainder (there is none of an infinity)
                        const float q = z * inverse, p = q < __builtin_huge_valf() ? fmaf(fmaf(-q, divisor, z), inverse, q) : q;
                        float y = z > 0.0f ? p : z * rho;
                        y = y - often * times;
                        y = times > 0.0f ? y - present : y;
                        x[k][e] = (c[e] != 0 ? y : z) + shift[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] = kept >> (k * 8 + e) & 1u ? x[k][e] : -__builtin_huge_valf();
            }
            if (mine == 8) store_tokens<DT>(yp + i * row, t, x[k]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < mine) {
                        if constexpr (DT == kDtBf16) ((uint16_t *)(yp + i * row))[t + e] = bf16_bits(x[k][e]);
                        else ((float *)(yp + i * row))[t + e] = x[k][e];
                    }
        }
    }
}

// Tokens into the counts: the prompt's set a flag, generated ones are added.
__global__ __launch_bounds__(256) void count_tokens_kernel(int32_t *count, const int32_t *tok, const int32_t *len, int V, int width, int prompt)
{
    const int b = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;   // (width is at most 2^30)
    if (j >= width || (len && j >= len[b])) return;
    const int v = tok[(long long)b * width + j];
    if (v < 0 || v >= V) return;
    int32_t *c = count + (long long)b * V + v;
    if (!prompt) atomicAdd(c, 1);
    else if (!(*c & kPromptFlag)) atomicOr(c, kPromptFlag);
}

}  // namespace stand
