// cache_four.hpp -- rows into a paged cache of 4 bits, and tokens out of a cache of either kind.
#pragma once
#include "cache_ops.hpp"
#include "mx4.hpp"

namespace stand {

// Where a cache's elements and scales are: strides of page, slot and head (and layer) in 16-byte chunks of the elements (8 of 16 bits, 32 of
// 4), and in bytes of the scales.
struct CachePlaces {
    char *k, *v;
    uint8_t *k_scale, *v_scale;
    long long layer, page, slot, head, scale_layer, scale_page, scale_slot, scale_head;
    int page_shift, pages;
};

constexpr int kFourUnit = 8;          // elements of a thread's part of a head on the way in: 16 bytes of 16-bit numbers, a quarter of a block
constexpr int kReadUnit = 16;         // on the way out: 8 bytes of 4-bit numbers
// Positions of a workgroup: as many as make a part for each thread.  (Two parts a thread, read before either is written: 223 us instead of
// 192 for the prompts below into the cache and out of it again, eight one after the other 237.)
STAND_BOTH int four_per_group(int row_units) { return (kCommitThreads + row_units - 1) / row_units; }

// ---- rows into 4 bits ---------------------------------------------------------------------------------------------------
// As cache_commit_kernel (cache_ops.hpp): row row[b][j] of trajectory b to slot slots[b][j], all layers.  A thread has 8 elements
// of a key and of a value: 16 bytes in, 4 out, and a block's four threads share its scale.  Bound by HBM with prompts (475 MB, 16 layers x
// 4 x up to 2100 rows of 8 heads of 128: 115 us, 4.1 TB/s), after a step by its trips to memory: count, slot and row, key and value
// (28 layers of 32 short paths: 6 us).
struct CommitFourArgs {
    const uint4 *k_rows, *v_rows;
    CachePlaces to;
    const int64_t *slots;
    const int32_t *row, *count;
    long long src_layer, src_batch, src_row, src_head;      // in 16-byte words
    long long slot_count;
    int rows, width, heads, units;                          // units: of one head
    int per_group;
};

template <bool F16>
__global__ __launch_bounds__(kCommitThreads) void cache_commit4_kernel(CommitFourArgs a)
{
    const int b = blockIdx.y, layer = blockIdx.z;
    const int n = commit_positions(a.count ? a.count[b] : a.width, a.width);
    const int row_units = a.heads * a.units;
    for (unsigned j0 = blockIdx.x * (unsigned)a.per_group; j0 < (unsigned)n; j0 += gridDim.x * (unsigned)a.per_group) {
        const int units = commit_words(n, j0, a.per_group, row_units);
        for (int i = threadIdx.x; i < units; i += kCommitThreads) {      // (a block's four threads come here together)
            const int j = (int)j0 + i / row_units, w = i % row_units;
            const int head = w / a.units, e = w % a.units;
            const long long slot = a.slots[(long long)b * a.width + j];
            const int r = a.row ? a.row[(long long)b * a.width + j] : j;
            if (slot < 0 || slot >= a.slot_count || r < 0 || r >= a.rows) continue;
            const long long src = layer * a.src_layer + b * a.src_batch + r * a.src_row + head * a.src_head + e;
            const long long page = slot >> a.to.page_shift, place = slot & ((1ll << a.to.page_shift) - 1);
            const long long dst = (layer * a.to.layer + page * a.to.page + place * a.to.slot + head * a.to.head) * 16 + 4 * e;
            const uint4 k = a.k_rows[src], v = a.v_rows[src];
            float x[8];
            uint32_t ks, vs;
            row_eight<F16>(k, x);
            *(uint32_t *)(a.to.k + dst) = mx4_quarter_block<F16>(x, ks);
            row_eight<F16>(v, x);
            *(uint32_t *)(a.to.v + dst) = mx4_quarter_block<F16>(x, vs);
            if (e % 4 == 0) {
                const long long sdst = layer * a.to.scale_layer + page * a.to.scale_page + place * a.to.scale_slot + head * a.to.scale_head + e / 4;
                a.to.k_scale[sdst] = (uint8_t)ks;
                a.to.v_scale[sdst] = (uint8_t)vs;
            }
        }
    }
}

// ---- tokens out of a cache -----------------------------------------------------------------------------------------------
// Token start[b] + j of trajectory b, j < count[b], to row j; tokens that no page in the cache has become zeros.  A thread writes 16
// elements of a key and of a value: of 16 bits it copies them, of 4 it makes them from 8 bytes and a scale.  (8 elements, a word of 4 bytes and
// a scale each: twice the time.)  Bound by HBM (the prompts above, 475 MB: 87 us, 5.5 TB/s).
struct ReadArgs {
    uint4 *k_rows, *v_rows;
    CachePlaces from;
    const int32_t *table, *start, *count;
    long long dst_layer, dst_batch, dst_row, dst_head;      // in 16-byte words
    int first_layer, rows, width, heads, units;
    int per_group;
};

enum ReadKind { kRead16, kReadBf16, kReadF16 };             // of 16 bits; of 4, as bf16 or fp16

template <ReadKind KIND>
__global__ __launch_bounds__(kCommitThreads) void cache_read_kernel(ReadArgs a)
{
    const int b = blockIdx.y, out_layer = blockIdx.z, layer = a.first_layer + out_layer;
    const int n = commit_positions(a.count ? a.count[b] : a.rows, a.rows);
    const int start = a.start ? a.start[b] : 0;
    const int row_units = a.heads * a.units;
    for (unsigned j0 = blockIdx.x * (unsigned)a.per_group; j0 < (unsigned)n; j0 += gridDim.x * (unsigned)a.per_group) {
        const int units = commit_words(n, j0, a.per_group, row_units);
        for (int i = threadIdx.x; i < units; i += kCommitThreads) {
            const int j = (int)j0 + i / row_units, w = i % row_units;
            const int head = w / a.units, e = w % a.units;
            const long long pos = (long long)start + j, at = pos >> a.from.page_shift;
            const int page = pos >= 0 && at < a.width ? a.table[(long long)b * a.width + at] : -1;
            const long long place = pos & ((1ll << a.from.page_shift) - 1);
            const long long dst = out_layer * a.dst_layer + b * a.dst_batch + j * a.dst_row + head * a.dst_head + 2 * e;
            uint4 k0{0, 0, 0, 0}, k1 = k0, v0 = k0, v1 = k0;
            if (page >= 0 && page < a.from.pages) {
                const long long src = (layer * a.from.layer + page * a.from.page + place * a.from.slot + head * a.from.head) * 16;
                if constexpr (KIND == kRead16) {
                    const uint4 *k = (const uint4 *)(a.from.k + src) + 2 * e, *v = (const uint4 *)(a.from.v + src) + 2 * e;
                    k0 = k[0]; k1 = k[1]; v0 = v[0]; v1 = v[1];
                } else {
                    constexpr bool F16 = KIND == kReadF16;
                    const long long ssrc = layer * a.from.scale_layer + page * a.from.scale_page + place * a.from.scale_slot + head * a.from.scale_head + e / 2;
                    const uint2 k = ((const uint2 *)(a.from.k + src))[e], v = ((const uint2 *)(a.from.v + src))[e];
                    const float ks = mx4_factor(a.from.k_scale[ssrc]), vs = mx4_factor(a.from.v_scale[ssrc]);
                    k0 = mx4_eight<F16>(k.x, ks); k1 = mx4_eight<F16>(k.y, ks);
                    v0 = mx4_eight<F16>(v.x, vs); v1 = mx4_eight<F16>(v.y, vs);
                }
            }
            a.k_rows[dst] = k0; a.k_rows[dst + 1] = k1;
            a.v_rows[dst] = v0; a.v_rows[dst + 1] = v1;
        }
    }
}

}  // namespace stand
