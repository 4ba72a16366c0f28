// row_turns.hpp -- heads of queries and keys normed and rotated by their rows' positions, in place, to other rows or on their way
// into a paged cache (of 16 bits or 4).
//
// For a head x of a row at position p:   y = w x / sqrt(mean(x^2) + eps)   (without a norm: y = x), then for each pair i of
// rotated elements, (a, b) = (y[i], y[i + half]) or (y[2 i], y[2 i + 1]):
//     a' = a cos(p, i) - b sin(p, i),   b' = a sin(p, i) + b cos(p, i)
// with cos and sin from the caller's table.  All of it in fp64, rounded to fp32 and from there to the type that is written: the vector
// units do fp64 at the rate of fp32, sums of squares cannot overflow, and what a key becomes in 4 bits is the nearest value of the formula's whatever
// the order of the sums.
//
// A thread has 16 elements of a head, whole pairs of them (two pieces of 8 that lie half a rotation apart, or 16 in a row), so
// that pairs need no exchange; D / 16 lanes have a head and add up their squares.  Workgroups have queries, keys or values, not a
// mixture.  For 4 bits a key's elements change lanes through LDS, so that blocks are of neighbours.
#pragma once
#include "cache_four.hpp"

namespace stand {

struct TurnArgs {
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;                         // or NULL
    long long qs[3], ks[3], vs[3], qos[3], kos[3];   // batch, row, head strides in elements
    const float *turns;                              // [positions][2 * half]: cosines, sines
    const uint16_t *q_norm, *k_norm;
    double eps;
    int positions, half, neighbours;
    const int32_t *start, *count;                    // [B] or NULL (0; all rows)
    const int32_t *tok;                              // a tree's rows: [B][rows], < 0: not drafted; NULL: rows in a line
    const unsigned long long *anc;
    int anc_words;
    int rows, q_heads, kv_heads, q_groups, k_groups; // workgroups of a trajectory's queries, keys; the others have values
    const int64_t *slots;                            // [B][width]
    int width;
    long long slot_count;
    CachePlaces to;
};

enum TurnTarget { kTurnRows, kTurnCache16, kTurnCache4 };
constexpr int kTurnThreads = 256;
constexpr int turn_heads_of_group(int d) { return kTurnThreads / (d / 16); }

template <int D, bool F16, TurnTarget TO>
__global__ __launch_bounds__(kTurnThreads) void row_turns_kernel(TurnArgs args)
{
    const TurnArgs &a = args;
    constexpr int LANES = D / 16, ITEMS = kTurnThreads / LANES;
    const int b = blockIdx.y, t = threadIdx.x % LANES;
    int group = blockIdx.x;
    const bool is_q = group < a.q_groups;
    if (!is_q) group -= a.q_groups;
    const bool is_k = !is_q && group < a.k_groups;
    if (!is_q && !is_k) group -= a.k_groups;
    const int heads = is_q ? a.q_heads : a.kv_heads;
    const unsigned item = (unsigned)group * ITEMS + threadIdx.x / LANES;
    const int row = (int)(item / (unsigned)heads), head = (int)(item % (unsigned)heads);
    const int n = a.count ? commit_positions(a.count[b], a.rows) : a.rows;
    if (row >= n) return;
    long long pos = (a.start ? a.start[b] : 0) + (long long)row;
    if (TO == kTurnRows && a.tok) {
        if (a.tok[(long long)b * a.rows + row] < 0) return;
        int depth = -1;
        for (int i = 0; i < a.anc_words; ++i) depth += __popcll(a.anc[row * a.anc_words + i]);
        pos += depth - row;
    }
    long long slot = -1;
    if (TO != kTurnRows && !is_q) {
        slot = a.slots[(long long)b * a.width + row];
        if (slot < 0 || slot >= a.slot_count) slot = -1;
        if (slot < 0 && (!is_k || !a.k_out)) return;
    }
    const long long page = slot >> a.to.page_shift, place = slot & ((1ll << a.to.page_shift) - 1);
    const long long dst = (page * a.to.page + place * a.to.slot + head * a.to.head) * 16;
    const long long sdst = page * a.to.scale_page + place * a.to.scale_slot + head * a.to.scale_head + t / 2;

    float y[16];
    if (TO != kTurnRows && !is_q && !is_k) {         // values, as they are
        const uint4 *from = (const uint4 *)(a.v + b * a.vs[0] + row * a.vs[1] + head * a.vs[2]) + 2 * t;
        const uint4 v0 = from[0], v1 = from[1];
        if constexpr (TO == kTurnCache16) {
            ((uint4 *)(a.to.v + dst))[2 * t] = v0;
            ((uint4 *)(a.to.v + dst))[2 * t + 1] = v1;
        } else {
            row_eight<F16>(v0, y);
            row_eight<F16>(v1, y + 8);
            uint32_t s;
            ((uint2 *)(a.to.v + dst))[t] = mx4_half_block<F16>(y, s);
            if (!(t & 1)) a.to.v_scale[sdst] = (uint8_t)s;
        }
        return;
    }
    // this thread's two pieces of eight elements
    const int turned = a.half / 8;                   // threads whose pairs are rotated
    const bool turns = t < turned, apart = turns && !a.neighbours;
    const int first = apart ? t : 2 * t, second = apart ? t + turned : 2 * t + 1;
    const uint16_t *x = is_q ? a.q + b * a.qs[0] + row * a.qs[1] + head * a.qs[2] : a.k + b * a.ks[0] + row * a.ks[1] + head * a.ks[2];
    const uint4 x0 = ((const uint4 *)x)[first], x1 = ((const uint4 *)x)[second];
    float cs[16];
    if (turns) {
        const bool there = pos >= 0 && pos < a.positions;
        const float4 *c = (const float4 *)(a.turns + (there ? pos : 0) * 2 * a.half + 8 * t), *s = c + a.half / 4;
        const float4 c0 = c[0], c1 = c[1], s0 = s[0], s1 = s[1];
        const float v[16] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w, s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
        for (int i = 0; i < 16; ++i) cs[i] = there ? v[i] : __builtin_nanf("");
    }
    float f[16];
    row_eight<F16>(x0, f);
    row_eight<F16>(x1, f + 8);
    double z[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = f[i];
    const uint16_t *norm = is_q ? a.q_norm : a.k_norm;
    if (norm) {
        float w[16];
        row_eight<F16>(((const uint4 *)norm)[first], w);
        row_eight<F16>(((const uint4 *)norm)[second], w + 8);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fma(z[i], z[i], sum);
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) sum += __shfl_xor(sum, off);
        const double r = 1.0 / sqrt(sum * (1.0 / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] *= r * (double)w[i];
    }
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // (pairs: element i of both pieces, or two neighbours)
            const double p = a.neighbours ? z[2 * i] : z[i], q = a.neighbours ? z[2 * i + 1] : z[8 + i];
            const double c = cs[i], s = cs[8 + i];
            const double p1 = fma(p, c, -(q * s)), q1 = fma(p, s, q * c);
            y[i] = (float)p1;
            y[8 + i] = (float)q1;
        }
        if (a.neighbours) {
            float w[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) { w[2 * i] = y[i]; w[2 * i + 1] = y[8 + i]; }
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = w[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = (float)z[i];
    }
    const uint4 o0{row_two<F16>(y[0], y[1]), row_two<F16>(y[2], y[3]), row_two<F16>(y[4], y[5]), row_two<F16>(y[6], y[7])};
    const uint4 o1{row_two<F16>(y[8], y[9]), row_two<F16>(y[10], y[11]), row_two<F16>(y[12], y[13]), row_two<F16>(y[14], y[15])};
    uint16_t *out = is_q ? a.q_out + b * a.qos[0] + row * a.qos[1] + head * a.qos[2]
                         : a.k_out ? a.k_out + b * a.kos[0] + row * a.kos[1] + head * a.kos[2] : nullptr;
    if (out) {
        ((uint4 *)out)[first] = o0;
        ((uint4 *)out)[second] = o1;
    }
    if constexpr (TO == kTurnCache16) {
        if (is_k && slot >= 0) {
            ((uint4 *)(a.to.k + dst))[first] = o0;
            ((uint4 *)(a.to.k + dst))[second] = o1;
        }
    }
    if constexpr (TO == kTurnCache4) {
        __shared__ float4 lines[kTurnThreads * 4];
        if (is_k && slot >= 0) {
            float4 *line = lines + threadIdx.x / LANES * (D / 4);
            line[2 * first] = float4{y[0], y[1], y[2], y[3]};
            line[2 * first + 1] = float4{y[4], y[5], y[6], y[7]};
            line[2 * second] = float4{y[8], y[9], y[10], y[11]};
            line[2 * second + 1] = float4{y[12], y[13], y[14], y[15]};
            // (a head's lanes are in one wave, whose accesses of LDS are in order)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 l = line[4 * t + i];
                y[4 * i] = l.x; y[4 * i + 1] = l.y; y[4 * i + 2] = l.z; y[4 * i + 3] = l.w;
            }
            uint32_t s;
            ((uint2 *)(a.to.k + dst))[t] = mx4_half_block<F16>(y, s);
            if (!(t & 1)) a.to.k_scale[sdst] = (uint8_t)s;
        }
    }
}

}  // namespace stand
