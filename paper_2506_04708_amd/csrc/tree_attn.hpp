// tree_attn.hpp -- attention of the nodes of a drafted tree over a paged key/value cache and over their own ancestors.
#pragma once
#include "attn_plan.hpp"
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace stand {

// What the workgroup leaves whose share begins inside an item that the one before it began: who has the parts.
struct JoinRecord { int first, last, rows, unused; };

struct TreeAttnArgs {
    const uint16_t *q, *k_new, *v_new, *k_pool, *v_pool;
    uint16_t *out;
    const int32_t *len, *table, *draft_tok;
    const uint32_t *anc;                             // [N][anc_words] bit sets in 32-bit words
    long long *total;                                // workspace: units of the call
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

// Asynchronous copies from global memory to LDS: lane l's 16 (4) bytes go to `to` + 16 l (4 l).  They have no result register;
// whoever reads what they bring waits for them (wait_loads) first.  (As builtins they make the compiler wait for all of them
// before any read of LDS, also of another buffer.)
__device__ __forceinline__ void copy16_async(const void *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void copy4_async(const void *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory");
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

template <int D_, bool F16_, int WR_, int WK_, int SUB_>
struct AttnShape {
    static constexpr int D = D_, WR = WR_, WK = WK_, SUB = SUB_;
    static constexpr bool F16 = F16_;
    static constexpr int WAVES = WR * WK, THREADS = 64 * WAVES;
    static constexpr int TM = 32 * WR;                 // query rows of a tile
    static constexpr int KT = 32 * WK * SUB;           // keys of a stage
    static constexpr bool ALONE = WR == 1;             // every wave loads the keys that it alone uses
    static constexpr int NBUF = ALONE ? 2 : 3;
    static constexpr int ROW = 2 * D;                  // bytes of a key
    static constexpr int CPR = D / 8;                  // 16-byte chunks of a key
    static constexpr int KPI = 64 / CPR;               // keys of one copy instruction
    static constexpr int LOADERS = WAVES >= 8 ? 8 : WAVES;  // waves that load
    static constexpr int KW = KT / LOADERS;            // keys that each of them loads per stage
    static constexpr int COPIES = 2 * KW / KPI;
    static constexpr int STAGE = 2 * KT * ROW;
    static constexpr int IDS = NBUF * STAGE;           // LDS: stages | page ids [4][LOADERS][64] | node list | scratch
    static constexpr int LIST = IDS + 4 * LOADERS * 256;
    static constexpr int MISC = LIST + 2048;
    static constexpr int BYTES = MISC + 256;
    static_assert(KW % KPI == 0 && KW >= KPI && KW <= 64, "a copy instruction brings whole keys of one wave");
    static_assert(!ALONE || LOADERS == WAVES, "every wave loads for itself");
    static_assert((WK - 1) * TM * (D + 2) * 4 <= NBUF * STAGE, "parts of the key waves are joined in the stages' memory");
    static_assert(8 * (kAttnMaxBatch + 1) <= NBUF * STAGE, "unit sums are made in the stages' memory");
    // 16-byte chunk c of key k stands at chunk c ^ swizzle(k): reads of one chunk of 16 keys (K) and of four chunks of four
    // keys (V) touch every bank once
    static __device__ __forceinline__ int swizzle_k(int k) { return D == 128 ? k & 15 : (k >> 1) & 7; }
    static __device__ __forceinline__ int swizzle_v(int k) { return D == 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2; }
};

// Units of work before each trajectory, prefix[0 .. B], in LDS: a unit is a stage of KT keys for one tile of rows and one
// key/value head.  Trajectory b has kv_heads * ceil(drafted * per_kv / TM) items of ceil(len / KT) + ceil(N / KT) units.
template <int TM, int KT, int THREADS>
__device__ __forceinline__ void unit_sums(const TreeAttnArgs &a, long long *prefix)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int p2 = 1;
    while (p2 < a.N && p2 < 64) p2 <<= 1;
    const int at_once = 64 / p2;                       // trajectories that a wave counts at once
    for (int b0 = wave * at_once; b0 < a.B; b0 += THREADS / 64 * at_once) {
        const int b = b0 + lane / p2;
        int count = 0;
        for (int u = lane % p2; u - lane % p2 < a.N; u += p2) {
            const bool there = b < a.B && u < a.N && a.draft_tok[(long long)b * a.N + u] >= 0;
            const unsigned long long bits = __ballot(there) >> (lane & ~(p2 - 1));
            count += __popcll(p2 == 64 ? bits : bits & ((1ull << p2) - 1));
        }
        if (b < a.B && lane % p2 == 0) prefix[b + 1] = item_units(a.len[b], (long long)a.width << a.page_shift, a.N, KT) * tree_items(count, a.per_kv, a.kv_heads, TM);
    }
    if (threadIdx.x == 0) prefix[0] = 0;
    __syncthreads();
    if (wave == 0) {
        long long base = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            long long x = b0 + lane < a.B ? prefix[b0 + lane + 1] : 0;
            for (int off = 1; off < 64; off <<= 1) {
                const long long y = __shfl_up(x, off);
                if (lane >= off) x += y;
            }
            x += base;
            if (b0 + lane < a.B) prefix[b0 + lane + 1] = x;
            base = __shfl(x, 63);
        }
    }
    __syncthreads();
}

template <typename S>
__global__ __launch_bounds__(S::THREADS, S::THREADS == 512 ? 2 : 1) void tree_attn_kernel(TreeAttnArgs a)
{
    constexpr int D = S::D, KT = S::KT, SUB = S::SUB, TM = S::TM, DT = D / 32, DC = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave % S::WR, wk = wave / S::WR, col = lane & 31, half = lane >> 5;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_char *)attn_lds);

    long long *sums = (long long *)attn_lds;
    unit_sums<TM, KT, S::THREADS>(a, sums);
    const long long total = sums[a.B];
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.total = total;
    // rows of nodes that were not drafted
    for (int r = blockIdx.x; r < a.B * a.N; r += a.groups)
        if (a.draft_tok[r] < 0)
            for (int i = threadIdx.x; i < a.kv_heads * a.per_kv * S::CPR; i += S::THREADS)
                *(uint4v *)(a.out + (r / a.N) * a.os[0] + (r % a.N) * a.os[1] + (i / S::CPR) * a.os[2] + i % S::CPR * 8) = uint4v{0, 0, 0, 0};
    const long long W = attn_groups(total, a.groups);
    // neighbours in the order of the work share an XCD (workgroups go round the eight of them in turn) and so its L2
    const int per_xcd = (int)((W + 7) / 8);
    const long long w = (long long)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if ((int)blockIdx.x / 8 >= per_xcd || w >= W) return;
    long long unit = group_start(w, total, W);
    const long long unit_end = group_start(w + 1, total, W);
    if (unit >= unit_end) return;
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
    const float c = a.scale * 1.4426950408889634f;
    // weights are at most 2^8 (where the running maximum is left behind); fp16 ones are scaled up so that few are subnormal
    constexpr float kUp = S::F16 ? 6.0f : 0.0f;

    while (unit < unit_end && b < a.B) {
        // ---- the item: trajectory, key/value head, tile of rows ----
        __syncthreads();
        uint16_t *list = (uint16_t *)(attn_lds + S::LIST);
        if (listed != b) {
            int base = 0;
            for (int u0 = 0; u0 < a.N; u0 += 64) {
                const int u = u0 + lane;
                const bool there = u < a.N && a.draft_tok[(long long)b * a.N + u] >= 0;
                const unsigned long long bits = __ballot(there);
                if (wave == 0 && there) list[base + __popcll(bits & ((1ull << lane) - 1))] = (uint16_t)u;
                base += __popcll(bits);
            }
            nodes = __builtin_amdgcn_readfirstlane(base);
            listed = b;
            __syncthreads();
        }
        if (nodes == 0) { ++b; continue; }             // nothing drafted: no units
        const long long most = (long long)a.width << a.page_shift;
        const int len = __builtin_amdgcn_readfirstlane((int)clamp_length(a.len[b], most));
        const int per_item = (int)item_units(len, most, a.N, KT), cache_units = (len + KT - 1) / KT;
        const int tiles = tree_items(nodes, a.per_kv, 1, TM);
        const int item = (int)((unit - b_start) / per_item);
        const int hk = item / tiles, tile = item % tiles;
        const long long item_start = b_start + (long long)item * per_item;
        const int u0 = (int)(unit - item_start);
        const int u1 = (int)(unit_end - item_start < per_item ? unit_end - item_start : per_item);
        bool leads = false;                            // this share is the second one of its first item
        if (first_item) {
            first_item = false;
            const long long from = group_of(item_start, total, W);
            leads = u0 > 0 && from == w - 1;
            if (threadIdx.x == 0)
                a.join[w] = JoinRecord{(int)from, (int)group_of(item_start + per_item - 1, total, W), leads ? min(TM, nodes * a.per_kv - tile * TM) : 0, 0};
        }
        const int rows = nodes * a.per_kv, row = tile * TM + wr * 32 + col;
        const bool busy = tile * TM + wr * 32 < rows;  // this wave has rows
        const int my_row = row < rows ? row : rows - 1;
        const int node = list[my_row / a.per_kv], head = hk * a.per_kv + my_row % a.per_kv;

        uint4v q[DC];
        {
            const uint16_t *qp = a.q + b * a.qs[0] + node * a.qs[1] + head * a.qs[2] + 8 * half;
#pragma unroll
            for (int i = 0; i < DC; ++i) q[i] = *(const uint4v *)(qp + 16 * i);
            // the wait for them belongs here: in the loop it would be one for the copies in flight as well
#pragma unroll
            for (int i = 0; i < DC; ++i) asm volatile("" : "+v"(q[i]));
        }
        float16v o[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = float16v{0};
        float m = -1e38f, l = 0.0f;                    // running maximum (scaled scores, base 2) and sum of the weights

        // this lane's first fragments inside a stage (chunk 0 of the keys, elements 0 .. 31 of the values); the others differ
        // in address bits that the swizzle only flips
        const uint32_t k_at = lds0 + (wk * SUB * 32 + col) * S::ROW + ((half ^ S::swizzle_k(col)) << 4);
        const int piece = lane & 3, j4 = (lane >> 2) & 3, dsub = (lane >> 4) & 1;
        const uint32_t v_at = lds0 + KT * S::ROW + (wk * SUB * 32 + 4 * half + j4) * S::ROW +
                              (((2 * dsub + (piece >> 1)) ^ S::swizzle_v(j4)) << 4) + (piece & 1) * 8;

        // ---- the units of this share: cached keys, then the tree's nodes; copies two stages ahead, page numbers two further ----
        const int n = u1 - u0, cached = cache_units - u0;       // units, those (if any) of the cache
        const int32_t *table = a.table + (long long)b * a.width;
        const int share = wave * S::KW;                         // this wave's keys of a stage (ALONE: those it uses)
        auto load_ids = [&](int i) {
            int key = (u0 + i) * KT + share + lane % S::KW;
            key = key < len ? key : len - 1;
            key = key > 0 ? key : 0;
            copy4_async(table + (key >> a.page_shift), __builtin_amdgcn_readfirstlane(lds0 + S::IDS + wave * 256 + (i & 3) * (S::LOADERS * 256)));
        };
        auto load_stage = [&](int i) {
            const uint32_t buf = lds0 + (i % S::NBUF) * S::STAGE + share * S::ROW;
            const int32_t *id = (const int32_t *)(attn_lds + S::IDS + (i & 3) * (S::LOADERS * 256) + wave * 256);
            const int ch = lane % S::CPR;
#pragma unroll
            for (int r = 0; r < S::KW / S::KPI; ++r) {
                const int at = r * S::KPI + lane / S::CPR, in_stage = share + at;
                const uint16_t *kp, *vp;
                if (i < cached) {
                    int key = (u0 + i) * KT + in_stage;
                    key = key < len ? key : len - 1;            // behind the end: the last key again, weighted with zero
                    const long long page = clamp_page(id[at], a.pages);
                    const long long from = page * a.pool_page + (key & ((1 << a.page_shift) - 1)) * a.pool_slot + hk * a.pool_head;
                    kp = a.k_pool + from;
                    vp = a.v_pool + from;
                } else {
                    int v = (i - cached) * KT + in_stage;
                    v = v < a.N ? v : a.N - 1;
                    kp = a.k_new + b * a.ks[0] + v * a.ks[1] + hk * a.ks[2];
                    vp = a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2];
                }
                copy16_async(kp + ((ch ^ S::swizzle_k(in_stage)) << 3), __builtin_amdgcn_readfirstlane(buf + r * S::KPI * S::ROW));
                copy16_async(vp + ((ch ^ S::swizzle_v(in_stage)) << 3), __builtin_amdgcn_readfirstlane(buf + KT * S::ROW + r * S::KPI * S::ROW));
            }
        };
        const bool loads = wave < S::LOADERS;
        if (loads) {
            load_ids(0); load_ids(1); load_ids(2);
            wait_loads<0>();
            load_stage(0);
            if (n > 1) { load_ids(3); load_stage(1); }
        }
        for (int i = 0; i < n; ++i) {
            const uint32_t off = (i % S::NBUF) * S::STAGE;
            if (i + 1 < n) wait_loads<S::COPIES + 1>();         // (the stage's own copies are all older than the newest that many)
            else wait_loads<0>();
            if constexpr (!S::ALONE) {
                group_barrier();                                // everyone's copies are there, and everyone is done with the stage before
                if (loads && i + 2 < n) { load_ids(i + 4); load_stage(i + 2); }
            }
            uint32_t word[SUB];                                 // keys of this wave that count, for this lane's query
            bool all = false, some;
            if (i < cached) {
                const int left = len - (u0 + i) * KT - wk * SUB * 32;
                all = left >= 32 * SUB;
                some = busy && left > 0;
#pragma unroll
                for (int t = 0; t < SUB; ++t) word[t] = left >= 32 * (t + 1) ? ~0u : (left <= 32 * t ? 0u : (1u << (left - 32 * t)) - 1u);
            } else {
                const int v0 = (i - cached) * KT;               // the unit's first node
                uint32_t any = 0;
#pragma unroll
                for (int t = 0; t < SUB; ++t) {
                    const int at = v0 / 32 + wk * SUB + t;
                    word[t] = busy && at * 32 < a.N ? a.anc[(long long)node * a.anc_words + at] : 0u;   // a node sees its ancestors and itself
                    any |= word[t];
                }
                some = __ballot(any != 0) != 0;
                // Values that are no finite numbers, of nodes that a row does not see, would reach it as 0 * infinity: they become
                // zeros here, and the rows that see them get them added below.
                uint32_t *odd = (uint32_t *)(attn_lds + S::MISC);
                if constexpr (S::ALONE) __syncthreads();        // (a wave may still read those of the unit before)
                if (threadIdx.x < KT / 32) odd[threadIdx.x] = 0;
                __syncthreads();
                for (int x = threadIdx.x; x < KT * S::CPR; x += S::THREADS) {
                    lds_uint4v *vp = (lds_uint4v *)(uintptr_t)(lds0 + off + KT * S::ROW + x * 16);
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
                        atomicOr(&odd[x / S::CPR / 32], 1u << (x / S::CPR & 31));
                    }
                }
                __syncthreads();
            }
            if (some) {
                // scores, weights, products with the values.  (The addresses are made opaque: what is added to them below is to
                // become part of the instructions.  The fences of the scheduler keep the reads of LDS ahead of their uses.)
                uint32_t ka = k_at + off, va = v_at + off;
                asm volatile("" : "+v"(ka), "+v"(va));
                float16v s[SUB];
                uint4v kf[SUB][DC];
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int x = 0; x < DC; ++x) kf[t][x] = *(const lds_uint4v *)(uintptr_t)((ka ^ (x << 5)) + t * 32 * S::ROW);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < SUB; ++t) {
                    s[t] = float16v{0};
#pragma unroll
                    for (int x = 0; x < DC; ++x) s[t] = mfma32<S::F16>(kf[t][x], q[x], s[t]);
                }
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
                if (!all) {
#pragma unroll
                    for (int t = 0; t < SUB; ++t) {
                        const uint32_t w4 = word[t] >> (4 * half);
#pragma unroll
                        for (int x = 0; x < 16; ++x) s[t][x] = w4 & (1u << (8 * (x / 4) + x % 4)) ? s[t][x] : -__builtin_huge_valf();
                    }
                }
                float top = s[0][0];
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int x = 0; x < 16; ++x) top = fmaxf(top, s[t][x]);
                top = other_half_max(top) * c;
                if (__ballot(top > m + 8.0f)) {                 // seldom after the first stages: the old maximum will do
                    const float next = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - next);
                    m = next;
                    l *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[d][x] *= f;
                }
                const float shift = kUp - m;
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
            }
            if (i >= cached && busy) {
                const uint32_t *odd = (const uint32_t *)(attn_lds + S::MISC);
                for (int t = 0; t < SUB; ++t)
                    for (uint32_t bits = odd[wk * SUB + t]; bits; bits &= bits - 1) {
                        // an infinity or NaN reaches the rows that see its node, whatever its weight
                        const int k = __builtin_ctz(bits), v = (i - cached) * KT + (wk * SUB + t) * 32 + k;
                        if (v >= a.N) break;
                        const bool sees = (a.anc[(long long)node * a.anc_words + v / 32] >> k) & 1u;
                        const uint16_t *vp = a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2] + 4 * half;
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const uint16_t h = vp[32 * d + 8 * (x / 4) + x % 4];
                                const float y = S::F16 ? (float)__builtin_bit_cast(_Float16, h) : __uint_as_float((uint32_t)h << 16);
                                if (sees && !(fabsf(y) < __builtin_huge_valf())) o[d][x] += y;
                            }
                    }
            }
            if constexpr (S::ALONE) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (i + 2 < n) { load_ids(i + 4); load_stage(i + 2); }
            }
        }

        // ---- the key waves' parts joined, then the rows' outputs or this workgroup's part of them ----
        l = other_half_sum(l);
        if constexpr (S::WK > 1) {
            __syncthreads();
            float *join = (float *)attn_lds;           // [WK - 1][WR][16 DT + 2][64]
            if (wk > 0) {
                float *to = join + ((wk - 1) * S::WR + wr) * (16 * DT + 2) * 64 + lane;
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
                for (int k = 0; k < S::WK - 1; ++k) next = fmaxf(next, join[(k * S::WR + wr) * (16 * DT + 2) * 64 + lane]);
                const float f = __builtin_amdgcn_exp2f(m - next);
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
#pragma unroll
                for (int k = 0; k < S::WK - 1; ++k) {
                    const float *from = join + (k * S::WR + wr) * (16 * DT + 2) * 64 + lane;
                    const float g = __builtin_amdgcn_exp2f(from[0] - next);
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
            if (u0 == 0 && u1 == per_item) {
                const float r = 1.0f / l;
                uint16_t *op = a.out + b * a.os[0] + node * a.os[1] + head * a.os[2] + 4 * half;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *(uint2 *)(op + 32 * d + 8 * i) = uint2{pack2<S::F16>(o[d][4 * i] * r, o[d][4 * i + 1] * r), pack2<S::F16>(o[d][4 * i + 2] * r, o[d][4 * i + 3] * r)};
            } else {
                float *to = a.part + (2 * w + (u0 == 0)) * (long long)TM * (D + 2);
                const int at = wr * 32 + col;
                if (half == 0) { to[at] = m; to[TM + at] = l; }
                to += 2 * TM + at * D + 4 * half;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) *(float4v *)(to + 32 * d + 8 * i) = float4v{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                if (leads && half == 0) a.place[w * TM + at] = b * a.os[0] + node * a.os[1] + head * a.os[2];
            }
        }
        unit = item_start + u1;
        if (unit == b_start + (long long)per_item * tiles * a.kv_heads) { b_start = unit; ++b; }
    }
}

// Rows of items that several workgroups took: their parts joined.  A task is four rows of an item, one for each wave, or one
// row whose parts the waves share where there are many.  Every workgroup sums up the records for itself and takes every
// gridDim.x-th task.  A lane holds D / 64 elements, and the weight of one part in 64.
constexpr int kJoinShared = 8;        // more parts: the waves share them
template <int D, int TM, bool F16>
__global__ __launch_bounds__(256) void tree_attn_join_kernel(TreeAttnArgs a)
{
    constexpr int E = D / 64;
    __shared__ int tasks[kAttnMaxGroups + 1], wave_sum[4];
    __shared__ float shared[4][D + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int W = (int)attn_groups(*a.total, a.groups), per = (W + 255) / 256;
    int sum = 0;
    for (int i = 0; i < per; ++i) {
        const int w = threadIdx.x * per + i;
        if (w < W) {
            const JoinRecord r = a.join[w];
            sum += r.last - r.first + 1 > kJoinShared ? r.rows : (r.rows + 3) / 4;
            tasks[w + 1] = sum;
        }
    }
    int before = sum;
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(before, off);
        if (lane >= off) before += y;
    }
    if (lane == 63) wave_sum[wave] = before;
    __syncthreads();
    before -= sum;
    for (int k = 0; k < wave; ++k) before += wave_sum[k];
    for (int i = 0; i < per; ++i)
        if (threadIdx.x * per + i < W) tasks[threadIdx.x * per + i + 1] += before;
    if (threadIdx.x == 0) tasks[0] = 0;
    __syncthreads();
    const int total = W > 0 ? tasks[W] : 0;
    for (int task = blockIdx.x; task < total; task += gridDim.x) {
        int lo = 0, hi = W - 1;                        // the record: last one with tasks[] <= task
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (tasks[mid] <= task) lo = mid; else hi = mid - 1;
        }
        const int w = __builtin_amdgcn_readfirstlane(lo), sub = task - tasks[w];
        const JoinRecord r = a.join[w];
        const bool share = r.last - r.first + 1 > kJoinShared;
        const int at = share ? sub : sub * 4 + wave;
        const int step = share ? 4 : 1, from = share ? r.first + wave : r.first;
        float acc[E], top = -1e38f, l = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.0f;
        const int parts = at < r.rows && from <= r.last ? (r.last - from) / step + 1 : 0;
        for (int k1 = 0; k1 < parts; k1 += 64) {
            const int here = min(parts - k1, 64), g = from + (k1 + min(lane, here - 1)) * step;
            const float *mine = a.part + (2 * g + (g == r.first)) * (long long)(TM * (D + 2));
            const float m = lane < here ? mine[at] : -1e38f, x = lane < here ? mine[TM + at] : 0.0f;
            float best = m;
            for (int off = 32; off > 0; off >>= 1) best = fmaxf(best, __shfl_xor(best, off));
            best = fmaxf(best, top);
            const float f = __builtin_amdgcn_exp2f(top - best), weight = __builtin_amdgcn_exp2f(m - best);
            top = best;
            l = fmaf(weight, x, l * f);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= f;
            for (int k0 = 0; k0 < here; k0 += 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = min(k0 + j, here - 1), gk = from + (k1 + k) * step;
                    const float *p = a.part + (2 * gk + (gk == r.first)) * (long long)(TM * (D + 2)) + 2 * TM + at * D + lane * E;
                    const float y = __shfl(weight, k);
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(k0 + j < here ? y : 0.0f, k0 + j < here ? p[e] : 0.0f, acc[e]);
                }
            }
        }
        for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
        if (share) {
            __syncthreads();                           // (the task before is done with them)
#pragma unroll
            for (int e = 0; e < E; ++e) shared[wave][lane * E + e] = acc[e];
            if (lane == 0) { shared[wave][D] = top; shared[wave][D + 1] = l; }
            __syncthreads();
            if (wave > 0) continue;
            const float best = fmaxf(fmaxf(shared[0][D], shared[1][D]), fmaxf(shared[2][D], shared[3][D]));
            l = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = __builtin_amdgcn_exp2f(shared[k][D] - best);
                l = fmaf(f, shared[k][D + 1], l);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(f, shared[k][lane * E + e], acc[e]);
            }
        }
        if (at >= r.rows) continue;
        uint16_t *o = a.out + a.place[(long long)w * TM + at] + lane * E;
        if constexpr (E == 2) *(uint32_t *)o = pack2<F16>(acc[0] / l, acc[1] / l);
        else o[0] = (uint16_t)pack2<F16>(acc[0] / l, 0.0f);
    }
}

}  // namespace stand
