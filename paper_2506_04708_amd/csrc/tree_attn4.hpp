// tree_attn4.hpp -- attention of the nodes of a drafted tree over a paged cache of 4 bits and over their own ancestors.
//
// The mathematics is tree_attn.hpp's: one pass over the keys with a running maximum, S^T = K Q^T and O^T = V^T P^T with 32x32x16
// products, weights rounded to the rows' type, sums in fp32.  A token's key and value are a quarter of the bytes; one instruction makes two numbers
// of the rows' type of two elements and their block's scale, exactly (mx4.hpp), and a wave needs 64 of them for 32 keys beside its 16 matrix
// instructions.  Two forms, by the rows that share a key/value head (serve_api.hip):
//
// Up to 64, every wave works by itself on 32 rows and a run of their keys: no barrier, no other wave's pace.  A lane has half of a key, D / 64
// blocks, straight from memory: a block's words, converted, are the left operand of four products, and the queries' elements are held in the
// same order.  Of a token's value a lane has half too; converted, it goes through 32 rows of LDS of the wave's own, from which the
// transposing reads take V^T.
//
// Above, the four waves of a workgroup have 32 rows each and the same keys (a team; a head's groups of 32 rows are shared out evenly over its
// teams).  Every thread converts one block of a unit into LDS for all, two units ahead of the products' reads of them in the third place of
// memory, and a step makes the scores of 32 keys beside the weights of the 32 before.  Two workgroups share a compute unit and do not wait for
// each other.  (Waves by themselves took 150 us when teams took 121 for the trees below: the vector units are the ones that are short, and every wave
// would convert everything; with all eight waves of a compute unit as one team, at one barrier, 133.)
//
// The tree comes first: the nodes that a wave's rows see, ancestors of a few nodes, are collected, so that most trees take one step of 32
// keys.  Their rows have 16 bits and take the first form's way without the conversions.
//
// Work is cut as attn_plan.hpp says, a share for every team that the chip holds; a unit is 32 keys (64 of heads of 64 in a team), the
// whole tree is one.  Beginnings count as START units (64 single tokens 214 us, with 3 225, with 10 216; 32 trees 122, 128, 123).
//
// Bound: decoding by HBM (1.08 GB of cache in 211 .. 217 us, 5.0 .. 5.1 TB/s; a torch copy reaches 5.0 counting both ways).  Trees by what a wave
// issues between its matrix instructions (32 trees of 64 nodes over 1000 .. 9000 tokens, 28 heads over 4, d 128: 125 .. 129 us for 70 GFLOP in passes one
// behind the other, 545 .. 560 TFLOP/s on rows as they are, where a large matrix product reaches 1253; over 16 bits, in turn with
// it, 132 and 126): a unit takes two workgroups about 1 us, of which the matrix units are busy for a half; of all clocks that compute units are at
// work, with waves that have no rows, beginnings and ends, for a third.  Short calls by the chain lengths -> shares -> nodes -> ancestors, page numbers -> keys, each
// a trip to memory.  Teams with d 128 have two registers too few: they are stored once an item and loaded behind its last key.
#pragma once
#include "mx4.hpp"
#include "tree_attn.hpp"

namespace stand {

struct TreeAttn4Args : TreeAttnArgs {                // k_pool, v_pool: blocks of 16 bytes; groups: shares
    const uint8_t *k_scale, *v_scale;                // pools of the blocks' scales, strides in bytes
    long long scale_page, scale_slot, scale_head;
    int workgroups;
};

// A form.  WR = 1: every wave of a workgroup works by itself.  WR = 4: the workgroup's waves have 32 rows each and the same keys.
template <int D_, bool F16_, int WR_>
struct Attn4Shape {
    static constexpr int D = D_, WR = WR_;
    static constexpr bool F16 = F16_, ALONE = WR == 1;
    static constexpr int WAVES = ALONE ? 4 : WR, THREADS = 64 * WAVES, MIN_WAVES = 2;
    static constexpr int TEAMS = WAVES / WR, TM = 32 * WR;   // shares of a workgroup, rows of one
    static constexpr int KT = ALONE || D == 128 ? 32 : 64, SUB = KT / 32;   // keys of a unit
    // units whose blocks are on their way (ALONE with two: decoding 220 us instead of 214, 60 000 tokens of 48 rows 62 instead of 56)
    static constexpr int AHEAD = ALONE ? 1 : 2;
    static constexpr int START = 6, HEAVY = 1, LIGHT = 1;
    static constexpr int ROW = 2 * D, CPR = D / 8;   // bytes and 16-byte chunks of a token's key or value
    static constexpr int BLOCKS = D / kMx4Block;     // of a key
    static constexpr int SUMS = (8 * (kAttnMaxBatch + 1) + 255) / 256 * 256;
    // LDS: 32 values of each wave, three units' keys and values in their place (unit sums before them) | drafted nodes of each team's
    // trajectory | nodes that a wave's rows see
    static constexpr int KEY_ROW = ROW + 16, KEYS = KT * KEY_ROW;
    static constexpr int VALUES = 32 * ROW, STAGE = KEYS + KT * ROW, ROWS = ALONE ? WAVES * VALUES : 3 * STAGE;
    static_assert(ROWS >= WAVES * VALUES, "a wave's values have room");
    static constexpr int LIST = ROWS > SUMS ? ROWS : SUMS, SEEN = LIST + TEAMS * 2048, SEEN_EACH = 2048 + 64, BYTES = SEEN + WAVES * SEEN_EACH;
    static __device__ __forceinline__ int tree_keys(int) { return 1; }
    static __device__ __forceinline__ int workgroups(const TreeAttn4Args &a) { return a.workgroups; }
    // Element of a head that a lane's first one of product x is.
    static __device__ __forceinline__ int element(int half, int x) { return ALONE ? D / 2 * half + 8 * x : 16 * x + 8 * half; }
    // Keys stand in rows of KEY_ROW bytes, so that a lane's chunks are a constant apart, and 16-byte chunk c of value k stands at chunk
    // c ^ swizzle_v(k): reads of one chunk of 16 keys, and the transposing ones of four chunks of four tokens, touch every one of 64 banks
    // once, and so do the places of 16 lanes' writes (a block of each of four or two keys; ALONE one chunk of 16 tokens).  But writes of 16 bytes go
    // eight lanes at a time to half of the banks, and of eight neighbours two meet in each: 16 clocks a write instead of 8, a quarter of what
    // LDS is busy for in teams (d 64: a sixth), two fifths ALONE.
    static __device__ __forceinline__ int swizzle_v(int k)
    {
        const int far = D == 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
        return far | (ALONE ? (k >> 2) & 3 : D == 128 ? k & 3 : (k >> 1) & 3);
    }
    static constexpr int EIGHT = ALONE ? 32 : 0;     // what it flips of an address eight tokens further on
};

// What a wave's lanes have written to LDS is read by others of them behind this (accesses of one wave are in order).
__device__ __forceinline__ void lanes_agree()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename S>
__global__ __launch_bounds__(S::THREADS, S::MIN_WAVES) void tree_attn4_kernel(TreeAttn4Args args)
{
    const TreeAttn4Args &a = fresh_args<TreeAttn4Args>();
    constexpr int D = S::D, DT = D / 32, DC = D / 16, HB = D / 64;   // tiles of the output, products of a score, blocks of half a key
    constexpr bool F16 = S::F16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;

    long long *sums = (long long *)attn_lds;
    unit_sums<S>(a, sums);
    const long long total = sums[a.B];
    const long long W = attn_groups(total, a.groups, S::START, S::HEAVY);
    const int wr = wave % S::WR, team = wave / S::WR, share_number = (int)blockIdx.x * S::TEAMS + team;
    if (wr == 0 && lane == 0 && share_number >= W) a.join[share_number] = JoinRecord{0, 0, 0, 0};   // (no share has this number)
    long long w;
    const bool has_share = share_of_team(blockIdx.x, team, S::TEAMS, W, w);
    long long unit = 0, unit_end = 0, b_start = 0;
    int b = 0;
    if (has_share) {
        unit = group_start(w, total, W);
        unit_end = group_start(w + 1, total, W);
        int lo = 0, hi = a.B - 1;                      // last b with sums[b] <= unit (and units of its own)
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (sums[mid] <= unit) lo = mid; else hi = mid - 1;
        }
        b = __builtin_amdgcn_readfirstlane(lo);
        b_start = sums[b];
    }
    __syncthreads();                                   // (the sums make room)
    int listed = -1, nodes = 0;
    bool first_item = true;
    const Exponent ex = exponent_of(a.scale);
    const float c = ex.c;
    uint16_t *const list = (uint16_t *)(attn_lds + S::LIST + team * 2048), *const seen = (uint16_t *)(attn_lds + S::SEEN + wave * S::SEEN_EACH);
    const uint32_t lds_begin = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_char *)attn_lds), lds0 = lds_begin + wave * S::VALUES;
    // where this lane's half of token `col` goes, its chunk 0 (chunk x: ^ x << 4), and where its reads of tokens 4 half + j4 and of
    // those eight further on begin
    const uint32_t put = lds0 + col * S::ROW + (((4 * HB * half) ^ S::swizzle_v(col)) << 4);
    const int piece = lane & 3, j4 = (lane >> 2) & 3, dsub = (lane >> 4) & 1;
    const uint32_t get = lds0 + (4 * half + j4) * S::ROW + (((2 * dsub + (piece >> 1)) ^ S::swizzle_v(4 * half + j4)) << 4) + (piece & 1) * 8;

    const int B = a.B;
    while (unit < unit_end && b < B) {
        // ---- the item: trajectory, key/value head, a team's rows ----
        const TreeAttn4Args &a = fresh_args<TreeAttn4Args>();
        if constexpr (!S::ALONE) {                     // (everyone is done with the item before)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            group_barrier();
        }
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
                    if (wr == 0 && there) list[base + __popcll(bits & ((1ull << lane) - 1))] = (uint16_t)u;
                    base += __popcll(bits);
                }
            }
            nodes = __builtin_amdgcn_readfirstlane(base);
            listed = b;
            if constexpr (S::ALONE) lanes_agree();
            else __syncthreads();
        }
        if (nodes == 0) { ++b; continue; }             // nothing drafted: no units
        const long long most = (long long)a.width << a.page_shift;
        const int len = __builtin_amdgcn_readfirstlane((int)clamp_length(a.len[b], most));
        const int cache_units = (len + S::KT - 1) / S::KT, units = cache_units + 1, per_item = units + S::START;   // (the first unit is the tree)
        const int all_rows = nodes * a.per_kv;
        const long long per_head = per_item * head_weight(all_rows, S::TM, S::HEAVY, S::LIGHT);
        const int heads_before = (int)quotient(unit - b_start, per_head);
        const long long head_start = b_start + heads_before * per_head;
        const int tile = (int)quotient(unit - head_start, per_item);
        const int row0 = tile_row(tile, all_rows, S::WR), rows = min(all_rows, tile_row(tile + 1, all_rows, S::WR));
        const int hk = (heads_before + b) % a.kv_heads;   // (not the same head of all trajectories at one time)
        const long long item_start = head_start + (long long)tile * per_item, item_end = item_start + per_item;
        const int u0 = (int)units_before(unit - item_start, 1, S::START, units), u1 = (int)units_before(unit_end - item_start, 1, S::START, units);
        if (u1 == 0) break;                            // the next one's
        bool leads = false;                            // this share is the second one of its first item
        if (first_item) {
            first_item = false;
            const long long from = first_group(item_start, total, W, S::START, 1);
            leads = u0 > 0 && from == w - 1;
            if (wr == 0 && lane == 0)                  // (every share comes here: none ends before its first item begins)
                a.join[w] = JoinRecord{(int)from, (int)group_of(item_end - 1, total, W), u0 > 0 ? rows - row0 : 0, 0};
        }
        const int row = row0 + wr * 32 + col, my_row = row < rows ? row : rows - 1;
        const int node = list[my_row / a.per_kv], head = hk * a.per_kv + my_row % a.per_kv;

        const bool busy = row0 + wr * 32 < rows;       // this wave has rows
        if constexpr (S::ALONE)
            if (!busy) __builtin_unreachable();
        float16v o[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = float16v{0};
        float m = -__builtin_huge_valf(), l = 0.0f;    // running maximum of the products with the keys, sum of the weights
        uint4v q[DC];
        {
            const uint16_t *qp = a.q + b * a.qs[0] + node * a.qs[1] + head * a.qs[2];
#pragma unroll
            for (int i = 0; i < DC; ++i) q[i] = *(const uint4v *)(qp + S::element(half, i));
        }
        // Scores of keys that are not among the first `left` of 32 count for nothing.
        auto mask_tail = [&](float16v &t, int left) {
            int from = left - 4 * half;
            asm volatile("" : "+v"(from));             // (compared with constants, not sixteen sums kept in registers)
#pragma unroll
            for (int x = 0; x < 16; ++x) t[x] = 8 * (x / 4) + x % 4 < from ? t[x] : -__builtin_huge_valf();
        };
        // Weights of the scores t of 32 keys, their products with the values in LDS.
        auto values = [&](float16v &t, uint32_t get) {
            uint4v vf[2][DT];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const short4v a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)((get ^ (d << 6)) + 16 * k * S::ROW));
                    const short4v a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)((get ^ (d << 6) ^ S::EIGHT) + (16 * k + 8) * S::ROW));
                    vf[k][d] = __builtin_bit_cast(uint4v, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            float top = t[0];
#pragma unroll
            for (int x = 1; x < 16; ++x) top = fmaxf(top, t[x]);
            float16v *const of[1] = {&t};
            const float shift = raise_row<F16>(ex, other_half_max(top), m, l, o, of);
            uint32_t p[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                p[x] = pack2<F16>(__builtin_amdgcn_exp2f(fmaf(t[2 * x], c, shift)), __builtin_amdgcn_exp2f(fmaf(t[2 * x + 1], c, shift)));
                l = add2<F16>(p[x], l);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] = mfma32<F16>(vf[k][d], uint4v{p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]}, o[d]);
        };

        // ---- the tree: the nodes that these rows see ----
        auto tree = [&]() {
            if (!busy || u0 != 0) return;
            const TreeAttn4Args &a = fresh_args<TreeAttn4Args>();
            const uint32_t *anc = a.anc + (long long)node * a.anc_words;
            int count = 0;
            for (int x0 = 0; 32 * x0 < a.N; x0 += 4) {
                uint32_t bits[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) bits[x] = anc[min(x0 + x, a.anc_words - 1)];
#pragma unroll
                for (int off = 1; off < 32; off <<= 1)
#pragma unroll
                    for (int x = 0; x < 4; ++x) bits[x] |= (uint32_t)__shfl_xor((int)bits[x], off);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t word = x0 + x < a.anc_words ? __builtin_amdgcn_readfirstlane(bits[x]) : 0u;
                    if (half == 0 && (word >> col & 1u)) seen[count + __popc(word & ((1u << col) - 1u))] = (uint16_t)(32 * (x0 + x) + col);
                    count += __popc(word);
                }
            }
            if (half == 0) seen[count + col] = 0;      // (the root, for what is left of the last 32)
            lanes_agree();
            for (int j0 = 0; j0 < count; j0 += 32) {
                const int v = seen[j0 + col];
                const uint16_t *kp = a.k_new + b * a.ks[0] + v * a.ks[1] + hk * a.ks[2];
                const uint16_t *vp = a.v_new + b * a.vs[0] + v * a.vs[1] + hk * a.vs[2] + D / 2 * half;
                // which of them this lane's row sees: bits of its 16 of the 32
                uint2 ids[4];
                uint32_t mine = 0, words[16];
#pragma unroll
                for (int g = 0; g < 4; ++g) ids[g] = *(const uint2 *)(seen + j0 + 8 * g + 4 * half);
                auto node_at = [&](int x) { return (x & 2 ? ids[x / 4].y : ids[x / 4].x) >> (16 * (x & 1)) & 0xFFFFu; };
#pragma unroll
                for (int x = 0; x < 16; ++x) words[x] = anc[node_at(x) / 32];
                uint4v kw[DC], vw[DC];
#pragma unroll
                for (int x = 0; x < DC; ++x) kw[x] = *(const uint4v *)(kp + S::element(half, x));
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < 16; ++x) mine |= (words[x] >> (node_at(x) & 31) & 1u) << (8 * (x / 4) + x % 4 + 4 * half);
                if (count - j0 < 32) mine &= (1u << (count - j0)) - 1u;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < DC; ++x) vw[x] = *(const uint4v *)(vp + 8 * x);
                // Values that are no finite numbers, of nodes that a row does not see, would reach it as 0 * infinity: they become
                // zeros, and the rows that see them get them added below.
                bool found = false;
#pragma unroll
                for (int x = 0; x < DC; ++x) {
                    constexpr uint32_t kExp = F16 ? 0x7C00u : 0x7F80u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = (vw[x][e] & kExp) == kExp, hi = ((vw[x][e] >> 16) & kExp) == kExp;
                        found |= lo | hi;
                        vw[x][e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
                    }
                    *(lds_uint4v *)(uintptr_t)(put ^ (x << 4)) = vw[x];   // (chunks D / 16 half + x)
                }
                const unsigned long long wild2 = __ballot(found && j0 + col < count);
                float16v t = float16v{0};
#pragma unroll
                for (int x = 0; x < DC; ++x) t = mfma32<F16>(kw[x], q[x], t);
#pragma unroll
                for (int x = 0; x < 16; ++x) t[x] = mine >> (8 * (x / 4) + x % 4 + 4 * half) & 1u ? t[x] : -__builtin_huge_valf();
                values(t, get);
                uint32_t wild = __builtin_amdgcn_readfirstlane((uint32_t)wild2 | (uint32_t)(wild2 >> 32));
                const uint32_t all = mine | (uint32_t)__shfl_xor((int)mine, 32);
                for (; wild; wild &= wild - 1) {
                    // an infinity or NaN reaches the rows that see its node, whatever its weight
                    const int j = __builtin_ctz(wild), u = seen[j0 + j];
                    const uint16_t *from = a.v_new + b * a.vs[0] + u * a.vs[1] + hk * a.vs[2] + 4 * half;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const uint16_t h = from[32 * d + 8 * (e / 4) + e % 4];
                            const float y = F16 ? (float)__builtin_bit_cast(_Float16, h) : __uint_as_float((uint32_t)h << 16);
                            if ((all >> j & 1u) && !(fabsf(y) < __builtin_huge_valf())) o[d][e] += y;
                        }
                }
            }
        };

        // ---- the cached keys of this share ----
        const int first = max(u0 - 1, 0), n = u1 - 1 - first;   // (the item's first unit is the tree)
        if constexpr (S::ALONE) tree();
        if (S::ALONE && n > 0) {
            const int32_t *table = a.table + (long long)b * a.width;
            const int page_shift = a.page_shift, pages = a.pages;
            const uint32_t pool_page = (uint32_t)(a.pool_page / kMx4Block), pool_slot = (uint32_t)(a.pool_slot / kMx4Block);
            const uint32_t scale_page = (uint32_t)(a.scale_page / (2 * HB)), scale_slot = (uint32_t)(a.scale_slot / (2 * HB));
            // scales in the order of their blocks: a block's number is its scale's
            const bool alike = pool_page == a.scale_page && pool_slot == a.scale_slot;
            const uint4v *k_pool = (const uint4v *)(a.k_pool + hk * a.pool_head / 4) + HB * half, *v_pool = (const uint4v *)(a.v_pool + hk * a.pool_head / 4) + HB * half;
            const uint8_t *k_scale = a.k_scale + hk * a.scale_head + HB * half, *v_scale = a.v_scale + hk * a.scale_head + HB * half;
            constexpr int AHEAD = S::AHEAD;
            uint4v kb[AHEAD][HB], vb[AHEAD][HB];
            uint32_t ks[AHEAD], vs[AHEAD];             // a byte for each block
            int page[AHEAD];
            auto key_of = [&](int i) { return min((first + i) * S::KT + col, len - 1); };   // behind the end: the last key again, weighted with zero
            auto page_of = [&](int i) { return table[key_of(i) >> page_shift]; };
            auto load = [&](int i, int u) {
                const int key = key_of(i);
                const uint32_t at = (uint32_t)clamp_page(page[u], pages), place = (uint32_t)(key & ((1 << page_shift) - 1));
                const unsigned long long from = at * pool_page + place * pool_slot;
                unsigned long long sfrom = from;
                if (!alike) sfrom = (unsigned long long)(at * scale_page + place * scale_slot) * (2 * HB);
#pragma unroll
                for (int r = 0; r < HB; ++r) {
                    kb[u][r] = k_pool[from + r];
                    vb[u][r] = v_pool[from + r];
                }
                if constexpr (HB == 2) {
                    ks[u] = *(const uint16_t *)(k_scale + sfrom);
                    vs[u] = *(const uint16_t *)(v_scale + sfrom);
                } else {
                    ks[u] = k_scale[sfrom];
                    vs[u] = v_scale[sfrom];
                }
                __builtin_amdgcn_sched_barrier(0);
                page[u] = page_of(i + AHEAD);          // (behind the blocks, and used when they have come)
                __builtin_amdgcn_sched_barrier(0);
            };
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) page[u] = page_of(u);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) load(u, u);
            auto unit_of_keys = [&](int i, int u) {
                float16v t = float16v{0};
#pragma unroll
                for (int r = 0; r < HB; ++r) {
                    const float kf = mx4_factor(ks[u] >> (8 * r) & 255u), vf = mx4_factor(vs[u] >> (8 * r) & 255u);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        t = mfma32<F16>(__builtin_bit_cast(uint4v, mx4_eight<F16>(kb[u][r][x], kf)), q[4 * r + x], t);
                        *(lds_uint4v *)(uintptr_t)(put ^ ((4 * r + x) << 4)) = __builtin_bit_cast(uint4v, mx4_eight<F16>(vb[u][r][x], vf));
                    }
                }
                load(i + AHEAD, u);
                const int left = len - (first + i) * S::KT;
                if (left < 32) mask_tail(t, left);
                values(t, get);
            };
            // (left in the middle, never skipped: the compiler counts the loads on their way along every path it sees)
            for (int i = 0;;) {
                bool done = false;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    unit_of_keys(i, u);
                    if (++i >= n) { done = true; break; }
                }
                if (done) break;
            }
        }
        if constexpr (!S::ALONE) {
            // every thread has a block of a unit: loaded AHEAD units before it is converted into LDS, which is one before the products
            const int32_t *table = a.table + (long long)b * a.width;
            const int page_shift = a.page_shift, pages = a.pages;
            const uint32_t pool_page = (uint32_t)(a.pool_page / kMx4Block), pool_slot = (uint32_t)(a.pool_slot / kMx4Block);
            const uint32_t scale_page = (uint32_t)(a.scale_page / S::BLOCKS), scale_slot = (uint32_t)(a.scale_slot / S::BLOCKS);
            // scales in the order of their blocks: a block's number is its scale's
            const bool alike = pool_page == a.scale_page && pool_slot == a.scale_slot;
            const uint4v *k_pool = (const uint4v *)(a.k_pool + hk * a.pool_head / 4), *v_pool = (const uint4v *)(a.v_pool + hk * a.pool_head / 4);
            const uint8_t *k_scale = a.k_scale + hk * a.scale_head, *v_scale = a.v_scale + hk * a.scale_head;
            constexpr int HALF = S::KT * S::BLOCKS;          // the first half of a unit's blocks are keys
            const int mine = (int)threadIdx.x % HALF, my_key = mine / S::BLOCKS, my_piece = mine % S::BLOCKS;
            const bool is_v = (int)threadIdx.x >= HALF;
            static_assert(2 * HALF == S::THREADS, "who has which block");
            const uint4v *const pool = (is_v ? v_pool : k_pool) + my_piece;
            const uint8_t *const scales = (is_v ? v_scale : k_scale) + my_piece;
            uint32_t to[4];                                  // where its four chunks go
#pragma unroll
            for (int x = 0; x < 4; ++x)
                to[x] = lds_begin + (is_v ? S::KEYS + my_key * S::ROW + (((4 * my_piece + x) ^ S::swizzle_v(my_key)) << 4)
                                          : my_key * S::KEY_ROW + 16 * (4 * my_piece + x));
            constexpr int AHEAD = S::AHEAD;
            uint4v block[AHEAD];
            uint32_t scale[AHEAD];
            // the first ones are asked for before the tree, whose trips to memory then are theirs too (128 trees of 128 nodes: 142 us
            // instead of 144; the other form has no registers for that)
            const int last = max(len - 1, 0);                // (with no key to come: any place of the cache)
            auto key_of = [&](int i) { return min((first + i) * S::KT + my_key, last); };   // behind the end: the last key again, weighted with zero
            auto page_of = [&](int i) { return table[key_of(i) >> page_shift]; };
            auto load = [&](int i, int page, uint4v &block, uint32_t &scale) {
                const int key = key_of(i);
                const uint32_t at = (uint32_t)clamp_page(page, pages), place = (uint32_t)(key & ((1 << page_shift) - 1));
                const unsigned long long from = at * pool_page + place * pool_slot;
                unsigned long long sfrom = from;
                if (!alike) sfrom = (unsigned long long)(at * scale_page + place * scale_slot) * S::BLOCKS;
                block = pool[from];
                scale = scales[sfrom];
            };
            auto store_word = [&](const uint4v &block, uint32_t scale, uint32_t stage, int x) {
                *(lds_uint4v *)(uintptr_t)(to[x] + stage) = __builtin_bit_cast(uint4v, mx4_eight<F16>(block[x], mx4_factor(scale)));
            };
            // (page numbers as far ahead of the blocks as those of the conversions: loads come back in order, and a wait for a
            // page number is one for all blocks before it)
            int page[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) page[u] = page_of(u);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) load(u, page[u], block[u], scale[u]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) page[u] = page_of(AHEAD + u);
            __builtin_amdgcn_sched_barrier(0);
            tree();
            if (n > 0) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                group_barrier();                                 // (everyone is done with the tree)
                const uint32_t k_at = lds_begin + col * S::KEY_ROW + 16 * half, v_at = get - lds0 + lds_begin + S::KEYS;
                // Two steps at a time, 32 keys apart: scores of these keys, in whose products' shadow the weights of the keys before are made; then
                // the products of those with their values, beside the search for these keys' maximum and the next unit's conversion.  A wave
                // issues in order, so vector instructions between the matrix instructions are what keeps both units busy.
                float top = -__builtin_huge_valf();
                auto step = [&](auto have_old, auto have_new, float16v &old, float16v &now, uint32_t k_off, uint32_t v_off, int left, auto fill) {
                    constexpr bool OLD = decltype(have_old)::value, NEW = decltype(have_new)::value;
                    constexpr int PER = 16 / DC, READS = 2 * DT / DC;
                    uint4v kf[DC], vf[2 * DT];
                    if constexpr (NEW) {
#pragma unroll
                        for (int x = 0; x < DC; ++x) kf[x] = *(const lds_uint4v *)(uintptr_t)(k_at + k_off + 32 * x);
                        now = float16v{0};
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    float shift = 0.0f;
                    float16v *const of[1] = {&old};
                    if constexpr (OLD) shift = raise_row<F16>(ex, other_half_max(top), m, l, o, of);
                    uint32_t p[8];
                    float e[2][PER];
#pragma unroll
                    for (int x = 0; x <= DC; ++x) {
                        if (x < DC) {
                            if constexpr (NEW) now = mfma32<F16>(kf[x], q[x], now);
                            if constexpr (OLD) {
#pragma unroll
                                for (int y = x * READS; y < (x + 1) * READS; ++y) {
                                    const uint32_t at = ((v_at + v_off) ^ (y % DT << 6)) + 16 * (y / DT) * S::ROW;
                                    const short4v a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)at);
                                    const short4v a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)(uintptr_t)(at + 8 * S::ROW));
                                    vf[y] = __builtin_bit_cast(uint4v, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                                }
#pragma unroll
                                for (int y = 0; y < PER; ++y) e[x & 1][y] = __builtin_amdgcn_exp2f(fmaf(old[x * PER + y], c, shift));
                            }
                        }
                        if constexpr (OLD)
                            if (x > 0) {
#pragma unroll
                                for (int y = 0; y < PER; y += 2) {
                                    const int at = ((x - 1) * PER + y) / 2;
                                    p[at] = pack2<F16>(e[(x - 1) & 1][y], e[(x - 1) & 1][y + 1]);
                                    l = add2<F16>(p[at], l);
                                    asm volatile("" : "+v"(p[at]), "+v"(l));   // (made here, not where they are used)
                                }
                            }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if constexpr (NEW) {
                        if (left < 32) mask_tail(now, left);
                    }
#pragma unroll
                    for (int y = 0; y < 2 * DT; ++y) {
                        const int k = y / DT;
                        if constexpr (OLD) o[y % DT] = mfma32<F16>(vf[y], uint4v{p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]}, o[y % DT]);
                        constexpr int EACH = 8 / DT;
                        if constexpr (NEW) {
#pragma unroll
                            for (int x = 0; x < EACH; ++x) top = y + x == 0 ? now[0] : fmaxf(top, now[y * EACH + x]);
                        }
                        fill(y);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                using Yes = std::true_type;
                using No = std::false_type;
                auto no_fill = [](int) {};
                float16v even = float16v{0}, odd = float16v{0};
#pragma unroll
                for (int x = 0; x < 4; ++x) store_word(block[0], scale[0], 0, x);
                load(AHEAD, page[0], block[0], scale[0]);
                __builtin_amdgcn_sched_barrier(0);
                page[0] = page_of(2 * AHEAD);
                __builtin_amdgcn_sched_barrier(0);
                uint32_t before = 0, here = 0, next = S::STAGE;  // places of the units: the one before, this one, the next
                auto unit_of_keys = [&](auto have_old, auto is_odd, int i, uint4v &block, uint32_t &scale, int &page) {   // block: of unit i + 1
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    group_barrier();                             // the unit's keys and values are there, those of two units before done with
                    const int left = len - (first + i) * S::KT;
                    auto fill = [&](int y) {                     // (past the last unit: that one's last key again)
                        if (y % (2 * DT / 4) == 0) store_word(block, scale, next, y / (2 * DT / 4));
                    };
                    if (!busy) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) store_word(block, scale, next, x);
                    } else if constexpr (S::SUB == 1) {
                        if constexpr (decltype(is_odd)::value) step(have_old, Yes{}, even, odd, here, before, left, fill);
                        else step(have_old, Yes{}, odd, even, here, before, left, fill);
                    } else {
                        step(have_old, Yes{}, odd, even, here, before + 32 * S::ROW, left, fill);
                        step(Yes{}, Yes{}, even, odd, here + 32 * S::KEY_ROW, here, left - 32, no_fill);
                    }
                    load(i + 1 + AHEAD, page, block, scale);
                    __builtin_amdgcn_sched_barrier(0);
                    page = page_of(i + 1 + 2 * AHEAD);
                    __builtin_amdgcn_sched_barrier(0);
                    before = here; here = next; next = next == 2 * S::STAGE ? 0 : next + S::STAGE;
                };
                unit_of_keys(No{}, No{}, 0, block[1 % AHEAD], scale[1 % AHEAD], page[1 % AHEAD]);
                static_assert(AHEAD % 2 == 0, "a place's units are all odd or all even");
                // (left in the middle, never skipped: the compiler counts the loads on their way along every path it sees)
                if (n > 1)
                    for (int i = 1;;) {
                        bool done = false;
#pragma unroll
                        for (int u = 0; u < AHEAD; u += 2) {
                            unit_of_keys(Yes{}, Yes{}, i, block[(u + 2) % AHEAD], scale[(u + 2) % AHEAD], page[(u + 2) % AHEAD]);
                            if (++i >= n) { done = true; break; }
                            unit_of_keys(Yes{}, No{}, i, block[(u + 3) % AHEAD], scale[(u + 3) % AHEAD], page[(u + 3) % AHEAD]);
                            if (++i >= n) { done = true; break; }
                        }
                        if (done) break;
                    }
                if (busy) {
                    if (S::SUB == 1 && (n & 1)) odd = even;
                    step(Yes{}, No{}, odd, even, 0, before + (S::SUB - 1) * 32 * S::ROW, 0, no_fill);
                }
            }
        }

        // ---- the rows' outputs, or this wave's part of them ----
        l = other_half_sum(l);
        m = fmaxf(m, kLowest);                         // (nothing seen: differences of maxima are numbers)
        if (busy && row < rows) {
            const TreeAttn4Args &a = fresh_args<TreeAttn4Args>();
            if (u0 == 0 && u1 == units) {
                const float r = 1.0f / l;
                uint16_t *op = a.out + b * a.os[0] + node * a.os[1] + head * a.os[2] + 4 * half;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *(uint2 *)(op + 32 * d + 8 * i) = uint2{pack2<F16>(o[d][4 * i] * r, o[d][4 * i + 1] * r), pack2<F16>(o[d][4 * i + 2] * r, o[d][4 * i + 3] * r)};
            } else {
                // (as the registers stand, so that every store is one run of 1 KiB)
                float *to = a.part + (2 * w + (u0 == 0)) * (long long)(S::TM * (D + 2));
                const int at = wr * 32 + col;
                if (half == 0) { to[at] = m; to[S::TM + at] = l; }
                float4v *to4 = (float4v *)(to + 2 * S::TM) + wr * (4 * DT * 64) + lane;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to4[(4 * d + i) * 64] = float4v{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                if (leads && half == 0) a.place[w * S::TM + at] = b * a.os[0] + node * a.os[1] + head * a.os[2];
            }
        }
        if (u1 < units) break;
        unit = item_end;
        if (unit == b_start + per_head * fresh_args<TreeAttn4Args>().kv_heads) { b_start = unit; ++b; }
    }
    zero_rows<S>(fresh_args<TreeAttn4Args>());         // (last: the first ones to be done have the time)
}

}  // namespace stand
