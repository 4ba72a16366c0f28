// attn_plan.hpp -- how stand_tree_attention's work is cut, the same on the host, in its two kernels and in tests.
//
// A unit is one stage of keys for one tile of query rows and one key/value head.  The units of all trajectories stand in one
// row; W workgroups take equal shares of it, so that trajectories of any lengths keep the whole chip busy.  A share that ends
// inside an item (a trajectory's tile of rows of one head) leaves a part of its sums, which a second kernel joins.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define STAND_BOTH __host__ __device__ __forceinline__
#else
#define STAND_BOTH inline
#endif

namespace stand {

constexpr int kAttnMaxBatch = 4096;   // trajectories of a call: their unit sums are made in LDS
// a / b of numbers that are not negative.  (A division of 64 bits costs the GPU half a microsecond, and these mostly fit 32.)
STAND_BOTH long long quotient(long long a, long long b)
{
    return (unsigned long long)(a | b) >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}
STAND_BOTH long long clamp_length(long long len, long long most) { return len < 0 ? 0 : (len > most ? most : len); }
STAND_BOTH int clamp_page(int page, int pages) { return page < 0 ? 0 : (page >= pages ? pages - 1 : page); }

// Units of one item: its cached keys, then the tree's nodes.
STAND_BOTH long long item_units(long long len, long long most, int nodes_of_tree, int keys)
{
    return (clamp_length(len, most) + keys - 1) / keys + (nodes_of_tree + keys - 1) / keys;
}
// A head's rows (drafted nodes times query heads that share its keys) are full tiles and what is left.  What a unit of a tile
// costs: `heavy`, or `light` where the tile fills no more than half of the waves.
STAND_BOTH int tile_weight(int rows, int tile_rows, int heavy, int light) { return 2 * rows > tile_rows ? heavy : light; }
// The weights of all tiles of a head together.
STAND_BOTH long long head_weight(int rows, int tile_rows, int heavy, int light)
{
    const int left = rows % tile_rows;
    return (long long)(rows / tile_rows) * heavy + (left ? tile_weight(left, tile_rows, heavy, light) : 0);
}
// What an item costs beside its units (nodes, queries, page numbers and first keys to wait for) counts as `start` units at its
// beginning, so that shares of many short items are no longer than others.  A share that would begin or end among them begins
// or ends at the item's beginning instead, one that would begin or end inside a unit does at the unit's beginning.
// Units of an item that lie before a place of the work, places counted from the item's beginning.
STAND_BOTH long long units_before(long long place, int weight, int start, long long units)
{
    if (place < 0) return 0;
    const long long u = quotient(place, weight) - start;
    return u < 0 ? 0 : (u > units ? units : u);
}
// Workgroups that get a share, of `groups` launched: no share is shorter than start + 1 units of the heaviest kind (with
// start + 2 shares oftener end in the next item: 3 .. 31 short trees 19 .. 36 us instead of 16 .. 31; 100 trees of 40 and of 224
// nodes would gain, 28 and 41 us instead of 31 and 44).
STAND_BOTH long long attn_groups(long long total, int groups, int start, int heavy)
{
    const long long w = quotient(total, heavy * (start + 1));
    return w >= groups ? groups : w > 0 ? w : total > 0;
}
STAND_BOTH long long group_start(long long w, long long total, long long W) { return quotient(w * total, W); }
// The last workgroup whose share would begin at or before a place.
STAND_BOTH long long group_of(long long place, long long total, long long W) { return quotient((place + 1) * W - 1, total); }
// The workgroup that has an item's first part.
STAND_BOTH long long first_group(long long item_start, long long total, long long W, int start, int weight)
{
    return group_of(item_start + (long long)(start + 1) * weight - 1, total, W);
}

}  // namespace stand
