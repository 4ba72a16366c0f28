// tree_attn.hpp -- attention of the nodes of a drafted tree over a paged key/value cache and over their own ancestors.
#pragma once
#include "attn_plan.hpp"
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace stand {

struct TreeAttnArgs {
    const uint16_t *q, *k_new, *v_new, *k_pool, *v_pool;
    uint16_t *out;
    const int32_t *len, *table, *draft_tok;
    const uint32_t *anc;                             // [N][anc_words] bit sets in 32-bit words
    long long *prefix;                               // workspace: [B + 1] units before each trajectory
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
    static constexpr int KW = KT / WAVES;              // keys that a wave loads per stage
    static constexpr int COPIES = 2 * KW / KPI;
    static constexpr int STAGE = 2 * KT * ROW;
    static constexpr int IDS = NBUF * STAGE;           // LDS: stages | page ids [4][WAVES][64] | node list | scratch
    static constexpr int LIST = IDS + 4 * WAVES * 256;
    static constexpr int MISC = LIST + 2048;
    static constexpr int BYTES = MISC + 256;
    static_assert(KW % KPI == 0 && (KPI <= KW), "a copy instruction brings whole keys of one wave");
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
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= a.B; b += S::THREADS) a.prefix[b] = sums[b];
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
        const int rows = nodes * a.per_kv, row = tile * TM + wr * 32 + col;
        const bool busy = tile * TM + wr * 32 < rows;  // this wave has rows
        const int my_row = row < rows ? row : rows - 1;
        const int node = list[my_row / a.per_kv], head = hk * a.per_kv + my_row % a.per_kv;

        uint4v q[DC];
        {
            const uint16_t *qp = a.q + b * a.qs[0] + node * a.qs[1] + head * a.qs[2] + 8 * half;
#pragma unroll
            for (int i = 0; i < DC; ++i) q[i] = *(const uint4v *)(qp + 16 * i);
        }
        float16v o[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = float16v{0};
        float m = -1e38f, l = 0.0f;                    // running maximum (scaled scores, base 2) and sum of the weights

        // addresses of this lane's fragments inside a stage
        uint32_t ka[DC], va[DT];
#pragma unroll
        for (int i = 0; i < DC; ++i) ka[i] = lds0 + (wk * SUB * 32 + col) * S::ROW + (((2 * i + half) ^ S::swizzle_k(col)) << 4);
        {
            const int piece = lane & 3, j = (lane >> 2) & 3, dsub = (lane >> 4) & 1;
#pragma unroll
            for (int i = 0; i < DT; ++i)
                va[i] = lds0 + KT * S::ROW + (wk * SUB * 32 + 4 * half + j) * S::ROW +
                        (((4 * i + 2 * dsub + (piece >> 1)) ^ S::swizzle_v(j)) << 4) + (piece & 1) * 8;
        }

        // one stage: scores, weights, products with the values; keys of which `seen` (nullptr: all of them) says nothing are left out
        auto stage = [&](uint32_t off, auto masked, const uint32_t (&word)[SUB]) {
            float16v s[SUB];
#pragma unroll
            for (int t = 0; t < SUB; ++t) {
                s[t] = float16v{0};
#pragma unroll
                for (int i = 0; i < DC; ++i) {
                    const uint4v kf = *(const __attribute__((address_space(3))) uint4v *)(uintptr_t)(ka[i] + off + t * 32 * S::ROW);
                    s[t] = mfma32<S::F16>(kf, q[i], s[t]);
                }
            }
            if constexpr (decltype(masked)::value) {
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[t][i] = (word[t] >> (8 * (i / 4) + i % 4 + 4 * half)) & 1u ? s[t][i] : -__builtin_huge_valf();
            }
            float top = s[0][0];
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
            top = other_half_max(top) * c;
            if (__ballot(top > m + 8.0f)) {            // seldom after the first stages: the old maximum will do
                const float next = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - next);
                m = next;
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
            }
            const float shift = kUp - m;
#pragma unroll
            for (int t = 0; t < SUB; ++t) {
                uint32_t p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = pack2<S::F16>(__builtin_amdgcn_exp2f(fmaf(s[t][2 * i], c, shift)), __builtin_amdgcn_exp2f(fmaf(s[t][2 * i + 1], c, shift)));
                    l = add2<S::F16>(p[i], l);
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint4v pf = {p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]};
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const uint32_t at = va[d] + off + (t * 32 + 16 * k) * S::ROW;
                        const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)at);
                        const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)(at + 8 * S::ROW));
                        const short vf[8] __attribute__((aligned(16))) = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                        o[d] = mfma32<S::F16>(__builtin_bit_cast(uint4v, vf), pf, o[d]);
                    }
                }
            }
        };

        // ---- cached keys: copies two stages ahead, their page numbers two further ----
        const int n = (u1 < cache_units ? u1 : cache_units) - u0;
        if (n > 0) {
            const int32_t *table = a.table + (long long)b * a.width;
            const uint32_t ids = lds0 + S::IDS + wave * 256;
            const int share = wave * S::KW;            // this wave's keys of a stage (ALONE: those it uses)
            auto load_ids = [&](int i) {
                int key = (u0 + i) * KT + share + lane % S::KW;
                key = key < len ? key : len - 1;
                copy4_async(table + (key >> a.page_shift), __builtin_amdgcn_readfirstlane(ids + (i & 3) * (S::WAVES * 256)));
            };
            auto load_stage = [&](int i) {
                const uint32_t buf = lds0 + (i % S::NBUF) * S::STAGE + share * S::ROW;
                const int32_t *id = (const int32_t *)(attn_lds + S::IDS + (i & 3) * (S::WAVES * 256) + wave * 256);
#pragma unroll
                for (int r = 0; r < S::KW / S::KPI; ++r) {
                    const int at = r * S::KPI + lane / S::CPR, in_stage = share + at;
                    int key = (u0 + i) * KT + in_stage;
                    key = key < len ? key : len - 1;   // behind the end: the last key again, weighted with zero
                    const long long page = clamp_page(id[at], a.pages);
                    const long long from = page * a.pool_page + (key & ((1 << a.page_shift) - 1)) * a.pool_slot + hk * a.pool_head;
                    const int ch = lane % S::CPR;
                    copy16_async(a.k_pool + from + ((ch ^ S::swizzle_k(in_stage)) << 3), __builtin_amdgcn_readfirstlane(buf + r * S::KPI * S::ROW));
                    copy16_async(a.v_pool + from + ((ch ^ S::swizzle_v(in_stage)) << 3), __builtin_amdgcn_readfirstlane(buf + KT * S::ROW + r * S::KPI * S::ROW));
                }
            };
            load_ids(0); load_ids(1); load_ids(2);
            wait_loads<0>();
            load_stage(0);
            if (n > 1) { load_ids(3); load_stage(1); }
            for (int i = 0; i < n; ++i) {
                if (i + 1 < n) wait_loads<S::COPIES + 1>();
                else wait_loads<0>();
                if constexpr (!S::ALONE) {
                    group_barrier();                   // everyone's copies are there, and everyone is done with the stage before
                    if (i + 2 < n) { load_ids(i + 4); load_stage(i + 2); }
                }
                const uint32_t off = (i % S::NBUF) * S::STAGE;
                if (busy) {
                    const int left = len - (u0 + i) * KT - wk * SUB * 32;
                    uint32_t word[SUB];
#pragma unroll
                    for (int t = 0; t < SUB; ++t) word[t] = left >= 32 * (t + 1) ? ~0u : (left <= 32 * t ? 0u : (1u << (left - 32 * t)) - 1u);
                    if (left >= 32 * SUB) stage(off, std::false_type{}, word);
                    else if (left > 0) stage(off, std::true_type{}, word);
                }
                if constexpr (S::ALONE) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if (i + 2 < n) { load_ids(i + 4); load_stage(i + 2); }
                }
            }
        }

        // ---- the tree's own keys: a node sees its ancestors and itself ----
        for (int un = u0 > cache_units ? u0 : cache_units; un < u1; ++un) {
            const int v0 = (un - cache_units) * KT;    // first node of the unit
            uint32_t *odd = (uint32_t *)(attn_lds + S::MISC);   // [KT / 32] nodes with a value that is no finite number
            __syncthreads();
            if (threadIdx.x < KT / 32) odd[threadIdx.x] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < KT * S::CPR; i += S::THREADS) {
                const int key = i / S::CPR, ch = i % S::CPR, v = v0 + key;
                uint4v kw = {0, 0, 0, 0}, vw = {0, 0, 0, 0};
                if (v < a.N && a.draft_tok[(long long)b * a.N + v] >= 0) {
                    kw = *(const uint4v *)(a.k_new + b * a.ks[0] + v * a.ks[1] + hk * a.ks[2] + 8 * ch);
                    vw = *(const uint4v *)(a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2] + 8 * ch);
                    constexpr uint32_t kExp = S::F16 ? 0x7C00u : 0x7F80u;
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {      // 0 * infinity would reach the rows that do not see this node
                        const bool lo = (vw[e] & kExp) == kExp, hi = ((vw[e] >> 16) & kExp) == kExp;
                        any |= lo | hi;
                        vw[e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
                    }
                    if (any) atomicOr(&odd[key / 32], 1u << (key & 31));
                }
                *(uint4v *)(attn_lds + key * S::ROW + ((ch ^ S::swizzle_k(key)) << 4)) = kw;
                *(uint4v *)(attn_lds + KT * S::ROW + key * S::ROW + ((ch ^ S::swizzle_v(key)) << 4)) = vw;
            }
            __syncthreads();
            if (busy) {
                uint32_t word[SUB];
                bool any = false;
#pragma unroll
                for (int t = 0; t < SUB; ++t) {
                    const int at = v0 / 32 + wk * SUB + t;
                    word[t] = at * 32 < a.N ? a.anc[(long long)node * a.anc_words + at] : 0u;
                    any |= word[t] != 0;
                }
                if (__ballot(any)) stage(0, std::true_type{}, word);
                for (int t = 0; t < SUB; ++t)
                    for (uint32_t bits = odd[wk * SUB + t]; bits; bits &= bits - 1) {
                        // what was taken out above: an infinity or NaN reaches the rows that see the node, whatever their weight
                        const int k = __builtin_ctz(bits), v = v0 + (wk * SUB + t) * 32 + k;
                        const bool sees = (word[t] >> k) & 1u;
                        const uint16_t *vp = a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2] + 4 * half;
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint16_t x = vp[32 * d + 8 * (i / 4) + i % 4];
                                const float y = S::F16 ? (float)__builtin_bit_cast(_Float16, x) : __uint_as_float((uint32_t)x << 16);
                                if (sees && !(fabsf(y) < __builtin_huge_valf())) o[d][i] += y;
                            }
                    }
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
            }
        }
        unit = item_start + u1;
        if (unit == b_start + (long long)per_item * tiles * a.kv_heads) { b_start = unit; ++b; }
    }
}

// Rows of items that several workgroups took: their parts joined.  Rows of nodes that were not drafted: zeros.  One wave per
// query head; a lane holds D / 64 elements, and the weight of one part in 64.
template <int D, int TM, int KT, bool F16>
__global__ __launch_bounds__(256) void tree_attn_join_kernel(TreeAttnArgs a)
{
    constexpr int E = D / 64;
    const int b = blockIdx.x / a.N, u = blockIdx.x % a.N, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t *tok = a.draft_tok + (long long)b * a.N;
    const int heads = a.kv_heads * a.per_kv;
    if (tok[u] < 0) {
        for (int h = blockIdx.y * 4 + wave; h < heads; h += gridDim.y * 4) {
            uint16_t *o = a.out + b * a.os[0] + u * a.os[1] + h * a.os[2] + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = 0;
        }
        return;
    }
    int rank = 0, nodes = 0;
    for (int v0 = 0; v0 < a.N; v0 += 64) {
        const int v = v0 + lane;
        const unsigned long long bits = __ballot(v < a.N && tok[v] >= 0);
        nodes += __popcll(bits);
        if (v0 + 64 <= u) rank += __popcll(bits);
        else if (v0 <= u) rank += __popcll(bits & ((1ull << (u - v0)) - 1));
    }
    const long long total = a.prefix[a.B], W = attn_groups(total, a.groups);
    const long long per_item = item_units(a.len[b], (long long)a.width << a.page_shift, a.N, KT);
    const int tiles = tree_items(nodes, a.per_kv, 1, TM);
    for (int h = blockIdx.y * 4 + wave; h < heads; h += gridDim.y * 4) {
        const int row = rank * a.per_kv + h % a.per_kv, at = row % TM;
        const long long start = a.prefix[b] + (h / a.per_kv * tiles + row / TM) * per_item;
        const long long first = group_of(start, total, W), last = group_of(start + per_item - 1, total, W);
        if (first == last) continue;                   // one workgroup had the whole item and wrote the row
        float acc[E], top = -1e38f, sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.0f;
        for (long long g0 = first; g0 <= last; g0 += 64) {
            const long long g = g0 + lane;
            const float *mine = a.part + (2 * (g <= last ? g : last) + (g == first)) * (long long)TM * (D + 2);
            const float m = g <= last ? mine[at] : -1e38f, l = g <= last ? mine[TM + at] : 0.0f;
            float best = m;
            for (int off = 32; off > 0; off >>= 1) best = fmaxf(best, __shfl_xor(best, off));
            best = fmaxf(best, top);
            const float f = __builtin_amdgcn_exp2f(top - best), weight = __builtin_amdgcn_exp2f(m - best);
            top = best;
            sum = fmaf(weight, l, sum * f);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= f;
            const int here = (int)(last - g0 < 63 ? last - g0 : 63) + 1;
            for (int k0 = 0; k0 < here; k0 += 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = k0 + j < here ? k0 + j : here - 1;
                    const float *p = a.part + (2 * (g0 + k) + (g0 + k == first)) * (long long)TM * (D + 2) + 2 * TM + at * D + lane * E;
                    const float x = k0 + j < here ? __shfl(weight, k) : 0.0f;
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(x, k0 + j < here ? p[e] : 0.0f, acc[e]);
                }
            }
        }
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        uint16_t *o = a.out + b * a.os[0] + u * a.os[1] + h * a.os[2] + lane * E;
        if constexpr (E == 2) *(uint32_t *)o = pack2<F16>(acc[0] / sum, acc[1] / sum);
        else o[0] = (uint16_t)pack2<F16>(acc[0] / sum, 0.0f);
    }
}

}  // namespace stand
