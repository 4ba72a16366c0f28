// tree_attn.hpp -- attention of the nodes of a drafted tree over a paged key/value cache and over their own ancestors.
//
// For a row (one node, one query head) and the keys t that it sees, c = scale * log2(e):
//     out = sum_t w_t value_t / sum_t w_t,    w_t = 2^(c * (s_t - m)),    s_t = query . key_t
// in one pass over the keys with a running m; any m gives the same quotient.  m is raised only where c * s passes c * m by more
// than 8: weights are then at most 2^8, sums stay far inside fp32, and the outputs are scaled anew a few times per row instead of
// at every maximum.  The exponent is one fused operation, c * s - (c * m rounded): the rounding is the same for all keys of a row,
// but where |c * m| passes 2^22 it would be a large number, so such rows take m from their scores first (raise_row).  Weights are
// rounded to the cache's type for the matrix cores and summed as rounded, so that numerator and denominator err together.  Scores,
// m, sums and outputs are fp32.
//
// Rows: drafted nodes are numbered through (a third of a tree is not drafted, and is not computed), and all query heads of a
// key/value head share its keys, so a tile has up to 256 rows of (node, head) that read a key once.  A wave has 32 of them.  It
// computes S^T = K Q^T with 32x32x16 products, so that a lane has one row and 16 of 32 keys: maximum and sum need one exchange
// between two lanes, and the weights stand where the second product O^T = V^T P^T wants its right operand, with the keys in
// another order; the values are read in that order (transposed by the LDS reads).  Queries, scores and weights stay in registers;
// what passes through LDS beside keys and values is page numbers, the nodes' ancestors and list, and parts of waves that have
// different keys of the same rows.
//
// Keys come in stages of 64 or 128 by asynchronous copies, page numbers two stages ahead of them, into a swizzled layout that
// both products read without bank conflicts.  Four stages of memory: two on their way, one in work, one whose values are
// still read.
//
// Work: trajectories differ in length a hundredfold, so tiles are cut by units of a stage, equal shares (by the units' costs) for
// every workgroup the chip holds (attn_plan.hpp); items that were cut are joined by a second kernel.  No sum is made by atomics:
// the same call gives the same bits.
//
// Bound: decoding by HBM (2.04 GB of cache in 354 us, 5.8 TB/s; a torch copy reaches 4.9 counting both ways); larger trees by
// what a wave issues between its matrix instructions (32 trees of 64 nodes over 1000 .. 9000 tokens, 28 heads over 4, d 128:
// 124 .. 134 us for 70 GFLOP, 525 .. 565 TFLOP/s on rows as they are, where a large matrix product reaches 1211); alone on a SIMD a
// step of 32 keys takes a wave 404 ns, of which its 16 matrix instructions are 262.  Short calls are bound by the chain lengths ->
// shares -> nodes -> page numbers -> keys, each a trip to memory: 10.8 us, and 2.2 us for the join.
#pragma once
#include "attn_plan.hpp"
#include "wave_ops.hpp"

#include <type_traits>

namespace stand {

// What a workgroup leaves whose share begins inside an item: who has the item's parts.  rows 0: nothing to join.
struct JoinRecord { int first, last, rows, unused; };

struct TreeAttnArgs {
    const uint16_t *q, *k_new, *v_new, *k_pool, *v_pool;
    uint16_t *out;
    const int32_t *len, *table, *draft_tok;
    const uint32_t *anc;                             // [N][anc_words] bit sets in 32-bit words
    JoinRecord *join;                                // workspace: [groups], then the rows' places in out, [groups][rows of a tile]
    long long *place;
    float *part;                                     // workspace: [2 * groups][rows of a tile][D + 2]
    long long qs[3], ks[3], vs[3], os[3];            // batch, node, head strides in elements
    long long pool_page, pool_slot, pool_head;
    float scale;
    int anc_words, B, N, per_kv, kv_heads, width, pages, page_shift, groups;
};

typedef short short4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) short4v lds_short4v;
typedef __attribute__((address_space(3))) uint4v lds_uint4v;
typedef __attribute__((address_space(3))) char lds_char;

extern __shared__ __attribute__((aligned(16))) char attn_lds[];

template <bool F16>
__device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c)
{
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Two weights rounded to the cache's type (nearest, ties to even), in one word.
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (F16) return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
    else return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// The two weights of a word, as rounded, added to a sum.
template <bool F16>
__device__ __forceinline__ float add2(uint32_t w, float s)
{
    if constexpr (F16) return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), f16x2{(_Float16)1.0f, (_Float16)1.0f}, s, false);
    else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, s, false);
}

__device__ __forceinline__ float other_half_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a row's weights are made with.  c and rise = 8 / c are the call's.
struct Exponent { float c, rise; };
__device__ __forceinline__ Exponent exponent_of(float scale)
{
    const float c = scale * 1.4426950408889634f;
    return Exponent{c, 8.0f / c};
}
// weights are at most 2^8 (where the running maximum is left behind); fp16 ones are scaled up so that few are subnormal
template <bool F16> constexpr float kUp = F16 ? 6.0f : 0.0f;
constexpr float kFarRow = 4194304.0f;   // 2^22: c * m is rounded by at most a quarter
constexpr float kLowest = -3.402823466e+38f;

// What c * m is rounded by in a row's shift: nothing where the row is far.
template <bool F16>
__device__ __forceinline__ float shift_error(const Exponent &e, float m)
{
    const float shift = fmaf(-m, e.c, kUp<F16>), off = fmaf(m, e.c, shift) - kUp<F16>;
    return fabsf(shift) > kFarRow ? 0.0f : off;
}
// What sums made with a maximum `from` are multiplied by where they join those made with `to`, as an exponent.  (c * (from - to)
// alone would be off by what the shifts were rounded by, an eighth of a weight at 2^21.)  `to` is no less than `from`, and one of
// them is finite.
template <bool F16>
__device__ __forceinline__ float lowered(const Exponent &e, float from, float to)
{
    return (from - to) * e.c + (shift_error<F16>(e, to) - shift_error<F16>(e, from));
}

// The running maximum m of a lane's row before the products with the values of the scores s[0 .. NS), whose largest one is `top`:
// -> the shift of their exponents, c * s + shift.  m is raised, and the sum l and outputs o are scaled, where `top` passes it by more
// than `rise`; m begins at -infinity.  Rows with |c * m| > 2^22 (nothing but -infinity seen among them) come here with every stage
// and get differences s - m for scores.  Seldom after the first stages: the old maximum will do.
template <bool F16, int NS, int DT>
__device__ __forceinline__ float raise_row(const Exponent &e, float top, float &m, float &l, float16v (&o)[DT], float16v *const (&s)[NS])
{
    float shift = fmaf(-m, e.c, kUp<F16>);
    if (__ballot(top > m + e.rise || fabsf(shift) > kFarRow)) {
        const float next = fmaxf(m, top), f = __builtin_amdgcn_exp2f(next > m ? lowered<F16>(e, m, next) : 0.0f);
        m = next;
        l *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int x = 0; x < 16; ++x) o[d][x] *= f;
        shift = fmaf(-m, e.c, kUp<F16>);
        const bool far = fabsf(shift) > kFarRow;
        const float from = far && m > -__builtin_huge_valf() ? m : 0.0f;
        shift = far ? kUp<F16> : shift;
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
            for (int x = 0; x < 16; ++x) (*s[k])[x] -= from;
    }
    return shift;
}

// Asynchronous copies from global memory to LDS: lane l's 16 (4) bytes go to `to` + 16 l (4 l).  They have no result register;
// whoever reads what they bring waits for them (wait_loads) first.  `to` is in m0, which has to be set an instruction ahead of the
// copy.  (As builtins they make the compiler wait for all of them before any read of LDS, also of another buffer.)
__device__ __forceinline__ void copy16_async(const void *from, uint32_t to)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void copy4_async(const void *from, uint32_t to)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(to), "v"(from) : "memory");
}
template <int NEWER>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NEWER) : "memory");
}
__device__ __forceinline__ void group_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A form of the kernel: WR waves with 32 rows each times WK waves with SUB * 32 keys of a stage each.
template <int D_, bool F16_, int WR_, int WK_, int SUB_>
struct AttnShape {
    static constexpr int D = D_, WR = WR_, WK = WK_, SUB = SUB_;
    static constexpr bool F16 = F16_;
    static constexpr int WAVES = WR * WK, THREADS = 64 * WAVES;
    static constexpr int MIN_WAVES = 2;                // of a SIMD: 256 registers for each
    static constexpr int TM = 32 * WR;                 // query rows of a tile
    static constexpr int KT = 32 * WK * SUB;           // keys of a stage
    static constexpr bool ALONE = WR == 1;             // every wave loads the keys that it alone uses
    static constexpr int NBUF = ALONE ? 2 : 4;         // stages in LDS: two on their way, one in work, one whose values are still read
    // units that the beginning of an item costs, see attn_plan.hpp (128 trees of 128 nodes with heads of 64: 169 us, with 6 170, with 12
    // 173; 32 trees of 64 with heads of 128: 132 us, with 2 138, with 6 133, with 8 135)
    static constexpr int START = ALONE ? 2 : D == 64 ? 8 : 4;
    // cost of a unit whose waves of rows share the SIMDs, and of one with a wave each, which its keys' way into LDS bounds (336 rows
    // of 32 trees, a tile of 256 and one of 80: 133 us; by 2 : 1 142, 5 : 4 136, two tiles of 168 rows 141)
    static constexpr int HEAVY = WR == 8 ? 3 : 1, LIGHT = WR == 8 ? 2 : 1;
    static constexpr int ROW = 2 * D;                  // bytes of a key
    static constexpr int CPR = D / 8;                  // 16-byte chunks of a key
    static constexpr int KPI = 64 / CPR;               // keys of one copy instruction
    static constexpr int KW = KT / WAVES;              // keys that a wave loads per stage
    static constexpr int COPIES = 2 * KW / KPI;
    static constexpr int STAGE = 2 * KT * ROW;
    static constexpr int SUMS = (8 * (kAttnMaxBatch + 1) + 255) / 256 * 256;
    // LDS: stages (unit sums before them) | page numbers or ancestors, [8 stages][WAVES][64] | node list | values that are not finite
    static constexpr int IDS = NBUF * STAGE > SUMS ? NBUF * STAGE : SUMS;
    static constexpr int LIST = IDS + 8 * WAVES * 256;
    static constexpr int MISC = LIST + 2048;
    static constexpr int BYTES = MISC + WAVES * 128;
    static_assert(KW % KPI == 0 && KW >= KPI && KW <= 64, "a copy instruction brings whole keys of one wave");
    static_assert(SUB == 1 || SUB == 2, "a step reads the keys of the other one of two subtiles ahead");
    // a wave's part as its registers stand: 16 (D / 32) outputs, maximum and sum of every lane
    static constexpr int LANE_PART = 16 * (D / 32) + 2, KEY_PARTS = (WK - 1) * WR * LANE_PART * 64 * 4;
    static_assert(KEY_PARTS <= NBUF * STAGE, "parts of the key waves are joined in the stages' memory");
    // 16-byte chunk c of key k stands at chunk c ^ swizzle(k): reads of one chunk of 16 keys (K) and of four chunks of four
    // keys (V) touch every bank once
    static __device__ __forceinline__ int swizzle_k(int k) { return D == 128 ? k & 15 : (k >> 1) & 7; }
    static __device__ __forceinline__ int swizzle_v(int k) { return D == 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2; }
};

// Units of work before each trajectory, prefix[0 .. B], in LDS: a unit is a stage of KT keys for one tile of rows and one
// key/value head.  Trajectory b has kv_heads * ceil(drafted * per_kv / TM) items of START + ceil(len / KT) + ceil(N / KT) units.
// Every workgroup counts all drafted nodes for itself, up to 16 reads of a wave in flight (128 trees of 128 nodes: 7 us).
template <typename S>
__device__ __forceinline__ void unit_sums(const TreeAttnArgs &a, long long *prefix)
{
    constexpr int THREADS = S::THREADS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first_len = a.len[lane < a.B ? lane : 0];    // (asked for before it is needed)
    if (threadIdx.x == 0) prefix[0] = 0;
    int lg = 0;
    while (1 << lg < a.N && lg < 6) ++lg;
    // a wave counts 64 >> lg trajectories at once, or 64 nodes of one after the other
    const int sub = lane & ((1 << lg) - 1), turns = (a.B + (64 >> lg) - 1) >> (6 - lg);
    const int ahead = (int)(blockIdx.x * 5u % (unsigned)turns);   // (not all of them the same line of the L2 at one time)
    constexpr int WAVES = THREADS / 64;
    auto count = [&](auto at_a_time) {
        constexpr int K = decltype(at_a_time)::value;
        for (int x0 = wave; x0 < turns; x0 += WAVES * K) {
            int n[K] = {}, b[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int x = x0 + k * WAVES, g = x + ahead < turns ? x + ahead : x + ahead - turns;
                b[k] = x < turns ? (g << (6 - lg)) + (lane >> lg) : a.B;
            }
            for (int u = sub; u - sub < a.N; u += 64) {
                int tok[K];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const bool there = b[k] < a.B && u < a.N;
                    const int v = a.draft_tok[there ? b[k] * a.N + u : 0];   // (read by all: a branch would wait for each)
                    tok[k] = there ? v : -1;
                }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const unsigned long long bits = __ballot(tok[k] >= 0) >> (lane - sub);
                    n[k] += __popcll(lg == 6 ? bits : bits & ((1ull << (1 << lg)) - 1));
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (sub == 0 && b[k] < a.B) prefix[b[k] + 1] = n[k];
        }
    };
    if (turns <= WAVES) count(std::integral_constant<int, 1>{});
    else if (turns <= 8 * WAVES) count(std::integral_constant<int, 8>{});
    else count(std::integral_constant<int, 16>{});
    __syncthreads();
    if (wave == 0) {
        long long base = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            const int b = b0 + lane;
            long long x = 0;
            if (b < a.B) x = (S::START + item_units(b0 ? a.len[b] : first_len, (long long)a.width << a.page_shift, a.N, S::KT)) * head_weight((int)prefix[b + 1] * a.per_kv, S::TM, S::HEAVY, S::LIGHT) * a.kv_heads;
            for (int off = 1; off < 64; off <<= 1) {
                const long long y = __shfl_up(x, off);
                if (lane >= off) x += y;
            }
            x += base;
            if (b < a.B) prefix[b + 1] = x;
            base = __shfl(x, 63);
        }
    }
    __syncthreads();
}

// Rows of nodes that were not drafted: zeros, an equal number of rows for every workgroup.
template <typename S>
__device__ __forceinline__ void zero_rows(const TreeAttnArgs &a)
{
    const int lane = threadIdx.x & 63;
    const unsigned all = a.B * a.N, each = (all + a.groups - 1) / a.groups, r0 = min(all, blockIdx.x * each), r1 = min(all, r0 + each);
    for (unsigned x = r0; x < r1; x += 64) {
        unsigned long long gone = __ballot(x + lane < r1 && a.draft_tok[x + lane < r1 ? x + lane : r0] < 0);
        for (; gone; gone &= gone - 1) {
            const unsigned r = x + __builtin_ctzll(gone), b = r / (unsigned)a.N;
            uint16_t *row = a.out + b * a.os[0] + (r - b * a.N) * a.os[1];
            for (int i = threadIdx.x; i < a.kv_heads * a.per_kv * S::CPR; i += S::THREADS)
                *(uint4v *)(row + (i / S::CPR) * a.os[2] + i % S::CPR * 8) = uint4v{0, 0, 0, 0};
        }
    }
}

template <typename S>
__global__ __launch_bounds__(S::THREADS, S::MIN_WAVES) void tree_attn_kernel(TreeAttnArgs args)
{
    // (every phase reads the arguments it needs anew: all of them at once do not fit the scalar registers)
    const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
    constexpr int D = S::D, KT = S::KT, SUB = S::SUB, TM = S::TM, DT = D / 32, DC = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave % S::WR, wk = wave / S::WR, col = lane & 31, half = lane >> 5;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_char *)attn_lds);

    long long *sums = (long long *)attn_lds;
    unit_sums<S>(a, sums);
    const long long total = sums[a.B];
    const long long W = attn_groups(total, a.groups, S::START, S::HEAVY);
    if (threadIdx.x == 0 && (long long)blockIdx.x >= W) a.join[blockIdx.x] = JoinRecord{0, 0, 0, 0};   // (no share has this number)
    // neighbours in the order of the work share an XCD (workgroups go round the eight of them in turn) and so its L2
    const int per_xcd = (int)((W + 7) / 8);
    const long long w = (long long)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if ((int)blockIdx.x / 8 >= per_xcd || w >= W) {
        zero_rows<S>(a);
        return;
    }
    long long unit = group_start(w, total, W);
    const long long unit_end = group_start(w + 1, total, W);
    int b = 0;
    {
        int lo = 0, hi = a.B - 1;                      // last b with sums[b] <= unit (and units of its own)
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (sums[mid] <= unit) lo = mid; else hi = mid - 1;
        }
        b = __builtin_amdgcn_readfirstlane(lo);
    }
    long long b_start = sums[b];
    int listed = -1, nodes = 0;
    bool first_item = true;
    const Exponent ex = exponent_of(a.scale);
    const float c = ex.c;

    const int B = a.B;
    while (unit < unit_end && b < B) {
        // ---- the item: trajectory, key/value head, tile of rows ----
        const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        group_barrier();                               // (not the fence of __syncthreads: it waits for the outputs' stores)
        uint16_t *list = (uint16_t *)(attn_lds + S::LIST);
        if (listed != b) {
            int base = 0;
            for (int u0 = 0; u0 < a.N; u0 += 256) {
                int tok[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) tok[k] = a.draft_tok[b * a.N + min(u0 + 64 * k + lane, a.N - 1)];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int u = u0 + 64 * k + lane;
                    const bool there = u < a.N && tok[k] >= 0;
                    const unsigned long long bits = __ballot(there);
                    if (wave == 0 && there) list[base + __popcll(bits & ((1ull << lane) - 1))] = (uint16_t)u;
                    base += __popcll(bits);
                }
            }
            nodes = __builtin_amdgcn_readfirstlane(base);
            listed = b;
            __syncthreads();
        }
        if (nodes == 0) { ++b; continue; }             // nothing drafted: no units
        const long long most = (long long)a.width << a.page_shift;
        const int len = __builtin_amdgcn_readfirstlane((int)clamp_length(a.len[b], most));
        const int units = (int)item_units(len, most, a.N, KT), cache_units = (len + KT - 1) / KT, per_item = units + S::START;
        const int all_rows = nodes * a.per_kv, full = all_rows / TM;
        const long long per_head = per_item * head_weight(all_rows, TM, S::HEAVY, S::LIGHT);
        const int heads_before = (int)quotient(unit - b_start, per_head);
        const long long head_start = b_start + heads_before * per_head;
        const int tile = min((int)quotient(unit - head_start, S::HEAVY * per_item), full);
        const int row0 = tile * TM, rows = min(all_rows, row0 + TM), weight = tile_weight(rows - row0, TM, S::HEAVY, S::LIGHT);
        // (trajectories begin with different heads: at one time the same head of all of them would use a part of the memory
        // channels, where a token's heads stand side by side)
        const int hk = (heads_before + b) % a.kv_heads;
        const long long item_start = head_start + (long long)tile * S::HEAVY * per_item, item_end = item_start + (long long)weight * per_item;
        const int u0 = (int)units_before(unit - item_start, weight, S::START, units), u1 = (int)units_before(unit_end - item_start, weight, S::START, units);
        if (u1 == 0) break;                            // the next one's
        bool leads = false;                            // this share is the second one of its first item
        if (first_item) {
            first_item = false;
            const long long from = first_group(item_start, total, W, S::START, weight);
            leads = u0 > 0 && from == w - 1;
            if (threadIdx.x == 0)                      // (every share comes here: none ends before its first item begins)
                a.join[w] = JoinRecord{(int)from, (int)group_of(item_end - 1, total, W), u0 > 0 ? rows - row0 : 0, 0};
        }
        const int row = row0 + wr * 32 + col;
        const bool busy = row0 + wr * 32 < rows;       // this wave has rows
        const int my_row = row < rows ? row : rows - 1;
        const int node = list[my_row / a.per_kv], head = hk * a.per_kv + my_row % a.per_kv;

        float16v o[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = float16v{0};
        float m = -__builtin_huge_valf(), l = 0.0f;    // running maximum of the products with the keys, sum of the weights

        // this lane's first fragments inside a stage (chunk 0 of the keys, elements 0 .. 31 of the values); the others differ
        // in address bits that the swizzle only flips
        const uint32_t k_at = lds0 + (wk * SUB * 32 + col) * S::ROW + ((half ^ S::swizzle_k(col)) << 4);
        const int piece = lane & 3, j4 = (lane >> 2) & 3, dsub = (lane >> 4) & 1;
        const uint32_t v_at = lds0 + KT * S::ROW + (wk * SUB * 32 + 4 * half + j4) * S::ROW +
                              (((2 * dsub + (piece >> 1)) ^ S::swizzle_v(j4)) << 4) + (piece & 1) * 8;

        // ---- the units of this share: cached keys, then the tree's nodes; copies two stages ahead, page numbers two further ----
        const int n = u1 - u0, cached = cache_units - u0;       // units, those (if any) of the cache
        const int32_t *table = a.table + (long long)b * a.width;
        // (places in the cache are counted in 16-byte chunks: 32 bits reach over 64 GiB of keys or values of a layer)
        const uint16_t *k_pool = a.k_pool + hk * a.pool_head, *v_pool = a.v_pool + hk * a.pool_head;
        const uint32_t pool_page = (uint32_t)(a.pool_page / 8), pool_slot = (uint32_t)(a.pool_slot / 8);
        const int pages = a.pages, page_shift = a.page_shift;
        const int share = wave * S::KW;                         // this wave's keys of a stage (ALONE: those it uses)
        // page numbers of a stage's keys; of the tree's stages the words of this wave's rows' ancestors
        auto load_ids = [&](int i) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + S::IDS + wave * 256 + (i & 7) * (S::WAVES * 256));
            if (i < cached) {
                int key = (u0 + i) * KT + share + lane % S::KW;
                key = key < len ? key : len - 1;
                copy4_async(table + (key >> page_shift), to);
            } else {
                const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
                const int v = (i - cached) * KT + (wk * SUB + half % SUB) * 32;
                copy4_async(a.anc + (long long)node * a.anc_words + (v < a.N ? v / 32 : 0), to);
            }
        };
        constexpr int LOADS = S::KW / S::KPI;
        auto load_cached = [&](int i) {
            const uint32_t buf = lds0 + (i % S::NBUF) * S::STAGE + share * S::ROW;
            const int32_t *id = (const int32_t *)(attn_lds + S::IDS + (i & 7) * (S::WAVES * 256) + wave * 256);
            const int ch = lane % S::CPR;
            int page[LOADS];
#pragma unroll
            for (int r = 0; r < LOADS; ++r) page[r] = id[r * S::KPI + lane / S::CPR];
#pragma unroll
            for (int r = 0; r < LOADS; ++r) {
                const int in_stage = share + r * S::KPI + lane / S::CPR;
                int key = (u0 + i) * KT + in_stage;
                key = key < len ? key : len - 1;                // behind the end: the last key again, weighted with zero
                const uint32_t from = (uint32_t)clamp_page(page[r], pages) * pool_page + (uint32_t)(key & ((1 << page_shift) - 1)) * pool_slot;
                copy16_async(k_pool + 8ull * (from + (ch ^ S::swizzle_k(in_stage))), __builtin_amdgcn_readfirstlane(buf + r * S::KPI * S::ROW));
                copy16_async(v_pool + 8ull * (from + (ch ^ S::swizzle_v(in_stage))), __builtin_amdgcn_readfirstlane(buf + KT * S::ROW + r * S::KPI * S::ROW));
            }
        };
        auto load_stage = [&](int i) {
            if (i < cached) {
                load_cached(i);
                return;
            }
            const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
            const uint32_t buf = lds0 + (i % S::NBUF) * S::STAGE + share * S::ROW;
            const int ch = lane % S::CPR;
            for (int r = 0; r < LOADS; ++r) {
                const int in_stage = share + r * S::KPI + lane / S::CPR;
                int v = (i - cached) * KT + in_stage;
                v = v < a.N ? v : a.N - 1;
                const uint16_t *kp = a.k_new + b * a.ks[0] + v * a.ks[1] + hk * a.ks[2], *vp = a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2];
                copy16_async(kp + ((ch ^ S::swizzle_k(in_stage)) << 3), __builtin_amdgcn_readfirstlane(buf + r * S::KPI * S::ROW));
                copy16_async(vp + ((ch ^ S::swizzle_v(in_stage)) << 3), __builtin_amdgcn_readfirstlane(buf + KT * S::ROW + r * S::KPI * S::ROW));
            }
        };
        uint4v q[DC];
        float16v s[SUB];
        // Scores of a stage.  (The addresses are made opaque: what is added to them below is to become part of the instructions.
        // The fences of the scheduler keep the reads of LDS ahead of their uses.)
        auto scores = [&](uint32_t off, bool all, const uint32_t (&word)[SUB]) {
            uint32_t ka = k_at + off;
            asm volatile("" : "+v"(ka));
#pragma unroll
            for (int t = 0; t < SUB; ++t) {
                uint4v kf[DC];
#pragma unroll
                for (int x = 0; x < DC; ++x) kf[x] = *(const lds_uint4v *)(uintptr_t)((ka ^ (x << 5)) + t * 32 * S::ROW);
                if (t == 0) __builtin_amdgcn_sched_barrier(0);
                s[t] = float16v{0};
#pragma unroll
                for (int x = 0; x < DC; ++x) s[t] = mfma32<S::F16>(kf[x], q[x], s[t]);
            }
            if (!all) {
#pragma unroll
                for (int t = 0; t < SUB; ++t) {
                    const uint32_t w4 = word[t] >> (4 * half);
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[t][x] = w4 & (1u << (8 * (x / 4) + x % 4)) ? s[t][x] : -__builtin_huge_valf();
                }
            }
        };
        // Weights of these scores, their products with the values.
        auto values = [&](uint32_t off) {
            uint32_t va = v_at + off;
            asm volatile("" : "+v"(va));
            uint4v vf[2][DT];
            auto read_values = [&](int t) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const uint32_t at = (va ^ (d << 6)) + (t * 32 + 16 * k) * S::ROW;
                        const short4v a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)at);
                        const short4v a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)(at + 8 * S::ROW));
                        vf[k][d] = __builtin_bit_cast(uint4v, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
            };
            read_values(0);
            __builtin_amdgcn_sched_barrier(0);
            float top = s[0][0];
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int x = 0; x < 16; ++x) top = fmaxf(top, s[t][x]);
            float16v *of[SUB];
#pragma unroll
            for (int t = 0; t < SUB; ++t) of[t] = &s[t];
            const float shift = raise_row<S::F16>(ex, other_half_max(top), m, l, o, of);
#pragma unroll
            for (int t = 0; t < SUB; ++t) {
                uint32_t p[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    p[x] = pack2<S::F16>(__builtin_amdgcn_exp2f(fmaf(s[t][2 * x], c, shift)), __builtin_amdgcn_exp2f(fmaf(s[t][2 * x + 1], c, shift)));
                    l = add2<S::F16>(p[x], l);
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[d] = mfma32<S::F16>(vf[k][d], uint4v{p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]}, o[d]);
                if (t + 1 < SUB) read_values(t + 1);
            }
        };
        // The same, 32 keys at a time and one step apart: scores of these keys, in whose products' shadow the weights of the keys
        // before are made; then the products of those with their values, beside the search for these keys' maximum, which the next
        // step begins with while its keys are read.  A wave issues in order, so vector instructions between the matrix instructions
        // are what keeps both units busy.  HAVE: the keys have been read by the step before; NEXT: read those 32 keys further on.
        uint4v kf[DC];
        float top = -__builtin_huge_valf();
        auto step = [&](auto have, auto next, float16v &old, float16v &t, uint32_t k_off, uint32_t v_off, bool all, uint32_t word) {
            uint32_t ka = k_at + k_off, va = v_at + v_off;
            asm volatile("" : "+v"(ka), "+v"(va));
            if constexpr (!decltype(have)::value) {
#pragma unroll
                for (int x = 0; x < DC; ++x) kf[x] = *(const lds_uint4v *)(uintptr_t)(ka ^ (x << 5));
                __builtin_amdgcn_sched_barrier(0);
            }
            float16v *const of[1] = {&old};
            const float shift = raise_row<S::F16>(ex, other_half_max(top), m, l, o, of);
            constexpr int PER = 16 / DC;               // weights beside a matrix instruction
            uint4v vf[2 * DT];
            t = float16v{0};
            uint32_t p[8];
            float e[2][PER];
#pragma unroll
            for (int x = 0; x <= DC; ++x) {
                if (x < DC) {
                    t = mfma32<S::F16>(kf[x], q[x], t);
                    constexpr int READS = 2 * DT / DC;
#pragma unroll
                    for (int y = x * READS; y < (x + 1) * READS; ++y) {
                        const uint32_t at = (va ^ (y % DT << 6)) + 16 * (y / DT) * S::ROW;
                        const short4v a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)at);
                        const short4v a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)(at + 8 * S::ROW));
                        vf[y] = __builtin_bit_cast(uint4v, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
#pragma unroll
                    for (int y = 0; y < PER; ++y) e[x & 1][y] = __builtin_amdgcn_exp2f(fmaf(old[x * PER + y], c, shift));
                }
                if (x > 0) {
#pragma unroll
                    for (int y = 0; y < PER; y += 2) {
                        const int at = ((x - 1) * PER + y) / 2;
                        p[at] = pack2<S::F16>(e[(x - 1) & 1][y], e[(x - 1) & 1][y + 1]);
                        l = add2<S::F16>(p[at], l);
                        asm volatile("" : "+v"(p[at]), "+v"(l));   // (made here, not where they are used)
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!all) {
                const uint32_t w4 = word >> (4 * half);
#pragma unroll
                for (int x = 0; x < 16; ++x) t[x] = w4 & (1u << (8 * (x / 4) + x % 4)) ? t[x] : -__builtin_huge_valf();
            }
            top = t[0];
#pragma unroll
            for (int y = 0; y < 2 * DT; ++y) {
                const int k = y / DT;
                o[y % DT] = mfma32<S::F16>(vf[y], uint4v{p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]}, o[y % DT]);
                constexpr int EACH = 8 / DT;
#pragma unroll
                for (int x = 0; x < EACH; ++x) top = fmaxf(top, t[y * EACH + x]);
                if constexpr (decltype(next)::value) {
                    constexpr int READS = DC / (2 * DT);
#pragma unroll
                    for (int x = y * READS; x < (y + 1) * READS; ++x) kf[x] = *(const lds_uint4v *)(uintptr_t)((ka ^ (x << 5)) + 32 * S::ROW);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        using Yes = std::true_type;
        using No = std::false_type;
        load_ids(0); load_ids(1); load_ids(2);
        {
            const uint16_t *qp = a.q + b * a.qs[0] + node * a.qs[1] + head * a.qs[2] + 8 * half;
#pragma unroll
            for (int i = 0; i < DC; ++i) q[i] = *(const uint4v *)(qp + 16 * i);
            // the wait for them belongs here: in the loop it would be one for the copies in flight as well
#pragma unroll
            for (int i = 0; i < DC; ++i) asm volatile("" : "+v"(q[i]));
        }
        wait_loads<0>();
        load_stage(0);
        if (n > 1) { load_ids(3); load_stage(1); }
        uint32_t *wild = (uint32_t *)(attn_lds + S::MISC);      // [WAVES][32]: nodes with a value that is no finite number, found by a wave
        if (lane < 32) wild[wave * 32 + lane] = 0;
        // A unit that has come: everyone's copies are there, two units ahead are on their way, the tree's values are finite.
        // -> the keys of this wave's subtile t that count for this lane's query: bits, `all` of them.
        auto arrive = [&](int i) {
            if (i + 1 < n) wait_loads<S::COPIES + 1>();         // (the unit's own copies are all older than the newest that many)
            else wait_loads<0>();
            if (i >= cached) {
                // Values that are no finite numbers, of nodes that a row does not see, would reach it as 0 * infinity: they become
                // zeros here, by the wave that loaded them, and the rows that see them get them added below.
                const uint32_t at = lds0 + (i % S::NBUF) * S::STAGE + KT * S::ROW + share * S::ROW;
                const int n_nodes = fresh_args<TreeAttnArgs>().N;
                for (int x = lane; x < S::KW * S::CPR; x += 64) {
                    lds_uint4v *vp = (lds_uint4v *)(uintptr_t)(at + x * 16);
                    uint4v vw = *vp;
                    constexpr uint32_t kExp = S::F16 ? 0x7C00u : 0x7F80u;
                    bool found = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = (vw[e] & kExp) == kExp, hi = ((vw[e] >> 16) & kExp) == kExp;
                        found |= lo | hi;
                        vw[e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
                    }
                    if (found) {
                        *vp = vw;
                        const int v = (i - cached) * KT + share + x / S::CPR;
                        if (v < n_nodes) atomicOr(&wild[wave * 32 + v / 32], 1u << (v & 31));
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            if constexpr (!S::ALONE) {
                group_barrier();                                // ... and everyone is done with the unit two before
                if (i + 2 < n) { load_ids(i + 4); load_stage(i + 2); }
            }
        };
        auto counting = [&](int i, int t, bool &all) {
            const int first = wk * SUB * 32 + t * 32;           // the subtile's first key in the unit
            all = false;
            if (i < cached) {
                const int left = len - (u0 + i) * KT - first;
                all = left >= 32;
                return left >= 32 ? ~0u : (left <= 0 ? 0u : (1u << left) - 1u);
            }
            const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
            const int v = (i - cached) * KT + first;            // a node sees its ancestors and itself
            const uint32_t word = ((const uint32_t *)(attn_lds + S::IDS + (i & 7) * (S::WAVES * 256) + wave * 256))[t * 32 + col];
            return busy && v < a.N ? word : 0u;
        };
        if constexpr (S::ALONE) {
            for (int i = 0; i < n; ++i) {
                const uint32_t off = (i % S::NBUF) * S::STAGE;
                arrive(i);
                bool all;
                const uint32_t word[1] = {counting(i, 0, all)};
                if (__ballot(word[0] != 0)) {
                    scores(off, all, word);
                    values(off);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (i + 2 < n) { load_ids(i + 4); load_stage(i + 2); }
            }
        } else {
            float16v even, odd;                               // scores of every other subtile: they change places, not registers
#pragma unroll
            for (int x = 0; x < 16; ++x) even[x] = -__builtin_huge_valf();
            // (before the first keys there is no weight at all, and values that are there: the first unit's own)
            uint32_t before = 0;
            // Units whose keys all count and behind which two more cached ones come, without a question asked: branches cost as much
            // here as arithmetic does.
            constexpr int AT_ONCE = SUB == 1 ? 2 : 1;           // (an even number of subtiles)
            const int whole = min(len / KT - u0, min(n, cached) - 2) / AT_ONCE * AT_ONCE;
            int first = 0;
            for (; first < whole; first += AT_ONCE) {
#pragma unroll
                for (int x = 0; x < AT_ONCE; ++x) {
                    const int i = first + x;
                    wait_loads<S::COPIES + 1>();
                    group_barrier();
                    load_ids(i + 4);
                    load_cached(i + 2);
                    const uint32_t off = (i % S::NBUF) * S::STAGE;
                    if (busy) {
#pragma unroll
                        for (int t = 0; t < SUB; ++t) {
                            const uint32_t here = off + t * 32 * S::ROW;
                            if (SUB > 1 && t == 0) step(No{}, Yes{}, even, odd, here, before, true, 0u);
                            else if (SUB > 1) step(Yes{}, No{}, odd, even, here, before, true, 0u);
                            else if (x % 2 == 0) step(No{}, No{}, even, odd, here, before, true, 0u);
                            else step(No{}, No{}, odd, even, here, before, true, 0u);
                            before = here;
                        }
                    }
                }
            }
            const int steps = n * SUB;
            for (int j = first > 0 ? first * SUB : 0; j <= steps; ++j) {   // (the last one: no new keys)
                const bool last = j == steps;
                if (!last && j % SUB == 0) arrive(j / SUB);
                if (!busy) continue;
                bool all = true;
                uint32_t word = 0, off = before;
                if (!last) {
                    word = counting(j / SUB, j % SUB, all);
                    off = (j / SUB % S::NBUF) * S::STAGE + j % SUB * 32 * S::ROW;
                }
                step(No{}, No{}, even, odd, off, before, all, word);
                even = odd;
                before = off;
            }
        }
        if (busy && u1 > cache_units) {
            const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
            for (int x = 0; x < (a.N + 31) / 32; ++x) {
                if (x % (KT / 32) / SUB != wk) continue;
                uint32_t bits = wild[wave * 32 + x];
                if constexpr (!S::ALONE)                        // (who alone uses its keys has found all there is in them)
#pragma unroll
                    for (int y = 0; y < S::WAVES; ++y) bits |= wild[y * 32 + x];
                for (; bits; bits &= bits - 1) {
                    // an infinity or NaN reaches the rows that see its node, whatever its weight
                    const int v = 32 * x + __builtin_ctz(bits);
                    const bool sees = (a.anc[(long long)node * a.anc_words + x] >> (v & 31)) & 1u;
                    const uint16_t *vp = a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2] + 4 * half;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const uint16_t h = vp[32 * d + 8 * (e / 4) + e % 4];
                            const float y = S::F16 ? (float)__builtin_bit_cast(_Float16, h) : __uint_as_float((uint32_t)h << 16);
                            if (sees && !(fabsf(y) < __builtin_huge_valf())) o[d][e] += y;
                        }
                }
            }
        }

        // ---- the key waves' parts joined, then the rows' outputs or this workgroup's part of them ----
        l = other_half_sum(l);
        m = fmaxf(m, kLowest);                         // (nothing seen: differences of maxima are numbers)
        if constexpr (S::WK > 1) {
            __syncthreads();
            float *join = (float *)attn_lds;           // [WK - 1][WR][LANE_PART][64]
            if (wk > 0) {
                float *to = join + ((wk - 1) * S::WR + wr) * S::LANE_PART * 64 + lane;
                to[0] = m; to[64] = l;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) to[(2 + 16 * d + i) * 64] = o[d][i];
            }
            __syncthreads();
            if (wk == 0) {
                float next = m;
#pragma unroll
                for (int k = 0; k < S::WK - 1; ++k) next = fmaxf(next, join[(k * S::WR + wr) * S::LANE_PART * 64 + lane]);
                const float f = __builtin_amdgcn_exp2f(lowered<S::F16>(ex, m, next));
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
#pragma unroll
                for (int k = 0; k < S::WK - 1; ++k) {
                    const float *from = join + (k * S::WR + wr) * S::LANE_PART * 64 + lane;
                    const float g = __builtin_amdgcn_exp2f(lowered<S::F16>(ex, from[0], next));
                    l = fmaf(g, from[64], l);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] = fmaf(g, from[(2 + 16 * d + i) * 64], o[d][i]);
                }
                m = next;
            }
        }
        if (wk == 0 && row < rows) {
            const TreeAttnArgs &a = fresh_args<TreeAttnArgs>();
            if (u0 == 0 && u1 == units) {
                const float r = 1.0f / l;
                uint16_t *op = a.out + b * a.os[0] + node * a.os[1] + head * a.os[2] + 4 * half;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *(uint2 *)(op + 32 * d + 8 * i) = uint2{pack2<S::F16>(o[d][4 * i] * r, o[d][4 * i + 1] * r), pack2<S::F16>(o[d][4 * i + 2] * r, o[d][4 * i + 3] * r)};
            } else {
                // (as the registers stand, so that every store is one run of 1 KiB)
                float *to = a.part + (2 * w + (u0 == 0)) * (long long)(TM * (D + 2));
                const int at = wr * 32 + col;
                if (half == 0) { to[at] = m; to[TM + at] = l; }
                float4v *to4 = (float4v *)(to + 2 * TM) + wr * (4 * DT * 64) + lane;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to4[(4 * d + i) * 64] = float4v{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                if (leads && half == 0) a.place[w * TM + at] = b * a.os[0] + node * a.os[1] + head * a.os[2];
            }
        }
        if (u1 < units) break;
        unit = item_end;
        if (unit == b_start + per_head * fresh_args<TreeAttnArgs>().kv_heads) { b_start = unit; ++b; }
    }
    zero_rows<S>(fresh_args<TreeAttnArgs>());          // (last: the first ones to be done have the time)
}

// Rows of items that several workgroups took: their parts joined (weights 2^(c * (m - largest m))), 32 rows (those of one wave) by a workgroup and in the layout of
// a wave's registers: lane l has the row l % 32 and every second group of four elements.  The workgroups of the item's second
// share take a quarter of the elements with each wave; where there are many parts, those of eight shares take an eighth each and
// their waves the parts in turn.  Bound by the trip record -> place -> parts: 2.3 us for a short tree, 14 us for the 17 MB of
// parts of 32 trees of 64 nodes (256 workgroups' shares, each up to two parts of 256 rows).
constexpr int kJoinShared = 8;        // more parts: shared
template <int D, int TM, bool F16>
__global__ __launch_bounds__(256) void tree_attn_join_kernel(TreeAttnArgs a)
{
    constexpr int GROUPS = D / 8;                      // groups of four elements of a lane
    constexpr int Q = GROUPS / 4, E = GROUPS / 8;      // a quarter of them, an eighth
    constexpr long long kSlot = TM * (D + 2);
    __shared__ float shared[4][4 * E + 2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = blockIdx.x, wr = blockIdx.y, at = wr * 32 + (lane & 31);
    const JoinRecord r = a.join[w];
    const Exponent ex = exponent_of(a.scale);
    if (wr * 32 >= r.rows) return;
    const int turn = w - r.first - 1;                  // 0: the item's second share
    const bool share = r.last - r.first + 1 > kJoinShared;
    if (turn >= (share ? 8 : 1)) return;
    const int row = at < r.rows ? at : r.rows - 1;
    const long long place = a.place[(r.first + 1ll) * TM + row];
    uint16_t *o = a.out + place + 4 * (lane >> 5);
    auto store = [&](int j, float4v x, float l) {      // group j: elements 32 (j / 4) + 8 (j % 4) + 4 (lane / 32) and the three behind
        if (at < r.rows) *(uint2 *)(o + 32 * (j / 4) + 8 * (j % 4)) = uint2{pack2<F16>(x[0] / l, x[1] / l), pack2<F16>(x[2] / l, x[3] / l)};
    };
    auto gather = [&](auto n, int group, int from, int step, float4v *acc, float &top, float &l) {
        constexpr int COUNT = decltype(n)::value, AT_ONCE = 16 / COUNT;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) acc[i] = float4v{0, 0, 0, 0};
        for (int g0 = from; g0 <= r.last; g0 += AT_ONCE * step) {
            float m[AT_ONCE], x[AT_ONCE];
            float4v p[AT_ONCE][COUNT];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {        // (past the last one: that one again, with no weight)
                const int g = min(g0 + k * step, r.last);
                const float *slot = a.part + (2 * g + (g == r.first)) * kSlot;
                m[k] = slot[at]; x[k] = slot[TM + at];
#pragma unroll
                for (int i = 0; i < COUNT; ++i) p[k][i] = ((const float4v *)(slot + 2 * TM))[(wr * GROUPS + group + i) * 64 + lane];
            }
            float best = top;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) best = fmaxf(best, m[k]);
            const float f = __builtin_amdgcn_exp2f(lowered<F16>(ex, top, best));
            top = best;
            l *= f;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) acc[i] = acc[i] * f;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                if (g0 + k * step > r.last) continue;
                const float y = __builtin_amdgcn_exp2f(lowered<F16>(ex, m[k], best));
                l = fmaf(y, x[k], l);
#pragma unroll
                for (int i = 0; i < COUNT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(y, p[k][i][e], acc[i][e]);
            }
        }
    };
    float top = kLowest, l = 0.0f;
    if (!share) {
        float4v acc[Q];
        gather(std::integral_constant<int, Q>{}, wave * Q, r.first, 1, acc, top, l);
#pragma unroll
        for (int i = 0; i < Q; ++i) store(wave * Q + i, acc[i], l);
        return;
    }
    float4v acc[E];
    gather(std::integral_constant<int, E>{}, turn * E, r.first + wave, 4, acc, top, l);
    shared[wave][4 * E][lane] = top;
    shared[wave][4 * E + 1][lane] = l;
#pragma unroll
    for (int i = 0; i < 4 * E; ++i) shared[wave][i][lane] = acc[i / 4][i % 4];
    __syncthreads();
    if (wave >= E) return;
    // wave i: its group of the eighth, over the four waves' parts
    const float best = fmaxf(fmaxf(shared[0][4 * E][lane], shared[1][4 * E][lane]), fmaxf(shared[2][4 * E][lane], shared[3][4 * E][lane]));
    float4v x = {0, 0, 0, 0};
    l = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(lowered<F16>(ex, shared[k][4 * E][lane], best));
        l = fmaf(f, shared[k][4 * E + 1][lane], l);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(f, shared[k][4 * wave + e][lane], x[e]);
    }
    store(turn * E + wave, x, l);
}

}  // namespace stand
