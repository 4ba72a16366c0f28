// row_turns.hpp -- heads of queries and keys normed and rotated by their rows' positions, in place, to other rows or on their way
// into a paged cache (of 16 bits or 4).
//
// For a head x of a row at position p:   y = w x / sqrt(mean(x^2) + eps)   (without a norm: y = x), then for each pair i of
// rotated elements, (a, b) = (y[i], y[i + half]) or (y[2 i], y[2 i + 1]):
//     a' = a cos(p, i) - b sin(p, i),   b' = a sin(p, i) + b cos(p, i)
// with cos and sin from the caller's table.  All of it in fp64, rounded to fp32 and from there to the type that is written: sums of
// squares cannot overflow, and what a key becomes in 4 bits is the nearest value of the formula's whatever the order of the sums.  (An
// fp64 operation takes a SIMD 4.4 clocks where an fp32 one takes 2.6, a conversion 4.5: with four waves on it, eight independent chains each.)
//
// A thread has 16 elements of a head, whole pairs of them (two pieces of 8 that lie half a rotation apart, or 16 in a row), so
// that pairs need no exchange; D / 16 lanes have a head and add up their squares.  Workgroups have queries, keys or values, not a
// mixture.  For 4 bits a key's elements change lanes through LDS, so that blocks are of neighbours.
//
// Bound by HBM with prompts (142 MB in and out, 4 x up to 2100 rows with 32 heads of queries, 8 of keys and values: 26 us, 5.5 TB/s).
// Trees are bound by how little is on its way at a time: a wave asks for what its row is decided by, then for rows and cosines, and
// has some 200 vector instructions for each head of its lanes, 139 of them fp64, and 150 for a row before them (128 trees of 128 nodes,
// 16/8 heads of 128, 85 MB: 25 .. 27 us; with its stores in the L2 and 132 instead of 128 registers, three waves of a SIMD instead of
// four, 31; one head for a thread, its conversions for each, 34; drafted nodes numbered through, so that waves are full, 32).
// 128 registers are too few for most forms: pairs half a rotation apart spill 2, keys into 16 bits 2 or (such pairs) 4, into 4 bits 6
// or 10, stored once a row and loaded again for every head.  Neighbouring pairs in rows spill none.
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
    int positions, half;
    const int32_t *start, *count;                    // [B] or NULL (0; all rows)
    const int32_t *tok;                              // a tree's rows: [B][rows], < 0: not drafted; NULL: rows in a line
    const unsigned long long *anc;
    int anc_words;
    int rows, q_heads, kv_heads, q_groups, k_groups; // workgroups of a trajectory's queries, keys; the others have values
    int q_step, k_step;                              // threads of a row's queries, of its keys (and values), in lots of D / 16
    const int64_t *slots;                            // [B][width]
    int width;
    long long slot_count;
    CachePlaces to;
};

enum TurnTarget { kTurnRows, kTurnRowsPast, kTurnCache16, kTurnCache4 };   // Past: past the caches (put_row), as the kinds behind it always
constexpr int kTurnThreads = 256;
constexpr int turn_heads_of_group(int d) { return kTurnThreads / (d / 16); }

// 1 / sqrt(x), off by a few steps of fp64: one step of third order on the instruction's 2^-25 or so.
__device__ __forceinline__ double inverse_root(double x)
{
    const double r = __builtin_amdgcn_rsq(x), e = fma(-x * r, r, 1.0);
    return x > 0.0 && x < __builtin_huge_val() ? fma(r * e, fma(e, 0.375, 0.5), r) : r;
}

// Rows that are written past the caches.  A tree's are where there are more than 64 MiB of them (stand_tree_rotate): the call by itself, on
// two sets of inputs in turn, then takes 28 us instead of 34 (128 trees of 128 nodes, 16/8 heads of 128; 62 and 79 for 256 trees); in place it takes
// 32 instead of 30.5; together with the attention behind it as long either way (322 and 322, 612 and 612; in place 326 and 326).
// Smaller trees' stay in the caches: past them the rotation and its attention take 153 us instead of 150 (128 trees of 128, 16/8 heads of 64).
//     Appended rows always are, whatever their number.  By itself an append of 4 prompts of 2100 (32/8 heads of 128) then takes 37 us into
// 16 bits and 45 into 4, instead of 51 and 60, in turn on two sets of inputs; in place 39 and 49 instead of 38 and 43.  What reads
// the rows next finds none of them in the caches: with a read of the tokens and a pass over the queries behind it 111 and 116 us instead of 102
// and 106 (in place 105 and 108 instead of 99 and 102), with a product of 70 GFLOP for that pass 133 and 137 instead of 130 and 137; four chunks of
// 1024 58 and 60 instead of 53 and 55.  Past 200 MB a call it is the better way behind which reader ever, by 1 .. 3 % (16 prompts of
// 2100: 378 and 400 us instead of 391 and 412).  For 64 single tokens it makes no difference (with their attention 42 and 30 us both ways).
template <bool PAST>
__device__ __forceinline__ void put_row(uint4 *to, const uint4 &v)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    if constexpr (PAST) __builtin_nontemporal_store(words{v.x, v.y, v.z, v.w}, (words *)to);
    else *to = v;
}

template <int D, bool F16, TurnTarget TO, bool NEIGHBOURS>
__global__ __launch_bounds__(kTurnThreads, 4) void row_turns_kernel(TurnArgs args)
{
    const TurnArgs &a = args;
    constexpr int LANES = D / 16, ITEMS = kTurnThreads / LANES;
    constexpr bool TREE = TO == kTurnRows || TO == kTurnRowsPast, PAST = TO != kTurnRows;
    const int b = blockIdx.y, t = threadIdx.x % LANES;
    int group = blockIdx.x;
    const bool is_q = group < a.q_groups;
    if (!is_q) group -= a.q_groups;
    const bool is_k = !is_q && group < a.k_groups;
    if (!is_q && !is_k) group -= a.k_groups;
    // heads step, 2 step, ... behind the first one
    const int heads = is_q ? a.q_heads : a.kv_heads, step = is_q ? a.q_step : a.k_step;
    const unsigned item = (unsigned)group * ITEMS + threadIdx.x / LANES;
    const int row = (int)(item / (unsigned)step), first_head = (int)(item % (unsigned)step);
    // (what a row is decided and placed by is asked for at once)
    long long pos = a.start ? a.start[b] : 0;
    if constexpr (TREE) {
        const int u = row < a.rows ? row : 0, tok = a.tok[(long long)b * a.rows + u];
        int depth = -1;
        for (int i = 0; i < a.anc_words; ++i) depth += __popcll(a.anc[u * a.anc_words + i]);
        if (row >= a.rows || tok < 0) return;
        pos += depth;
    } else {
        if (row >= (a.count ? commit_positions(a.count[b], a.rows) : a.rows)) return;
        pos += row;
    }
    long long slot = -1;
    if (!TREE && !is_q) {
        slot = a.slots[(long long)b * a.width + row];
        if (slot < 0 || slot >= a.slot_count) slot = -1;
        if (slot < 0 && (!is_k || !a.k_out)) return;
    }
    const long long page = slot >> a.to.page_shift, place = slot & ((1ll << a.to.page_shift) - 1);
    const long long dst = (page * a.to.page + place * a.to.slot) * 16, dst_head = a.to.head * 16;
    const long long sdst = page * a.to.scale_page + place * a.to.scale_slot + t / 2;

    float y[16];
    if (!TREE && !is_q && !is_k) {         // values, as they are
        for (int head = first_head; head < heads; head += step) {
            const uint4 *from = (const uint4 *)(a.v + b * a.vs[0] + row * a.vs[1] + head * a.vs[2]) + 2 * t;
            const uint4 v0 = from[0], v1 = from[1];
            char *to = a.to.v + dst + head * dst_head;
            if constexpr (TO == kTurnCache16) {
                put_row<PAST>((uint4 *)to + 2 * t, v0);
                put_row<PAST>((uint4 *)to + 2 * t + 1, v1);
            } else {
                row_eight<F16>(v0, y);
                row_eight<F16>(v1, y + 8);
                uint32_t s;
                ((uint2 *)to)[t] = mx4_half_block<F16>(y, s);
                if (!(t & 1)) a.to.v_scale[sdst + head * a.to.scale_head] = (uint8_t)s;
            }
        }
        return;
    }
    // this thread's two pieces of eight elements
    const int turned = a.half / 8;                   // threads whose pairs are rotated
    const bool turns = t < turned, apart = turns && !NEIGHBOURS;
    const int first = apart ? t : 2 * t, second = apart ? t + turned : 2 * t + 1;
    const long long x_head = is_q ? a.qs[2] : a.ks[2];
    const uint16_t *x = is_q ? a.q + b * a.qs[0] + row * a.qs[1] : a.k + b * a.ks[0] + row * a.ks[1];
    uint16_t *out = is_q ? a.q_out + b * a.qos[0] + row * a.qos[1] : a.k_out ? a.k_out + b * a.kos[0] + row * a.kos[1] : nullptr;
    const long long out_head = is_q ? a.qos[2] : a.kos[2];
    uint4 x0 = ((const uint4 *)(x + first_head * x_head))[first], x1 = ((const uint4 *)(x + first_head * x_head))[second];
    // cosines and sines of its pairs, weights of its elements: the same for all heads
    double cs[16], weight[16];
    if (turns) {
        const bool there = pos >= 0 && pos < a.positions;
        const float4 *c = (const float4 *)(a.turns + (there ? pos : 0) * 2 * a.half + 8 * t), *s = c + a.half / 4;
        const float4 c0 = c[0], c1 = c[1], s0 = s[0], s1 = s[1];
        const float v[16] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w, s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
        for (int i = 0; i < 16; ++i) cs[i] = there ? v[i] : __builtin_nanf("");
    }
    const uint16_t *norm = is_q ? a.q_norm : a.k_norm;
    if (norm) {
        float w[16];
        row_eight<F16>(((const uint4 *)norm)[first], w);
        row_eight<F16>(((const uint4 *)norm)[second], w + 8);
#pragma unroll
        for (int i = 0; i < 16; ++i) weight[i] = w[i];
    }
    for (int head = first_head; head < heads; head += step) {
        float f[16];
        row_eight<F16>(x0, f);
        row_eight<F16>(x1, f + 8);
        if (head + step < heads) {
            x0 = ((const uint4 *)(x + (head + step) * x_head))[first];
            x1 = ((const uint4 *)(x + (head + step) * x_head))[second];
        }
        double z[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = f[i];
        if (norm) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fma(z[i], z[i], sum);
#pragma unroll
            for (int off = 1; off < LANES; off <<= 1) sum += __shfl_xor(sum, off);
            const double r = inverse_root(fma(sum, 1.0 / D, a.eps));
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] *= r * weight[i];
        }
        if (turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (pairs: element i of both pieces, or two neighbours)
                constexpr int FAR = NEIGHBOURS ? 1 : 8, BY = NEIGHBOURS ? 2 : 1;
                const double p = z[BY * i], q = z[BY * i + FAR];
                y[BY * i] = (float)fma(p, cs[i], -(q * cs[8 + i]));
                y[BY * i + FAR] = (float)fma(p, cs[8 + i], q * cs[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = (float)z[i];
        }
        const uint4 o0{row_two<F16>(y[0], y[1]), row_two<F16>(y[2], y[3]), row_two<F16>(y[4], y[5]), row_two<F16>(y[6], y[7])};
        const uint4 o1{row_two<F16>(y[8], y[9]), row_two<F16>(y[10], y[11]), row_two<F16>(y[12], y[13]), row_two<F16>(y[14], y[15])};
        if (out) {
            put_row<PAST>((uint4 *)(out + head * out_head) + first, o0);
            put_row<PAST>((uint4 *)(out + head * out_head) + second, o1);
        }
        if (TREE || !is_k || slot < 0) continue;
        char *to = a.to.k + dst + head * dst_head;
        if constexpr (TO == kTurnCache16) {
            put_row<PAST>((uint4 *)to + first, o0);
            put_row<PAST>((uint4 *)to + second, o1);
        }
        if constexpr (TO == kTurnCache4) {
            __shared__ float4 lines[kTurnThreads * 4];
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
            ((uint2 *)to)[t] = mx4_half_block<F16>(y, s);
            if (!(t & 1)) a.to.k_scale[sdst + head * a.to.scale_head] = (uint8_t)s;
        }
    }
}

}  // namespace stand
