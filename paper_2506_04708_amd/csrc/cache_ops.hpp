// cache_ops.hpp -- the paged key/value cache between two target model passes: rows into their slots, and the pages of
// each trajectory (block tables, slot maps, the ring of free pages).  Everything these kernels decide by is on the device
// (accepted lengths, accepted nodes), so that a serving loop never waits for the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace stand {

// ---- rows into the cache ------------------------------------------------------------------------------------------------
// For every layer, trajectory b and j < count[b]: the keys and values of source row row[b][j] go to slot slots[b][j].  A slot
// is page * page_size + place in the page.  All strides are in 16-byte words.
struct CommitArgs {
    const uint4 *k_rows, *v_rows;
    uint4 *k_pool, *v_pool;
    const int64_t *slots;       // [B][width]
    const int32_t *row, *count; // [B][width] or NULL (row j), [B] or NULL (width)
    long long src_layer, src_batch, src_row, src_head;      // keys' and values' rows have the same strides
    long long pool_layer, pool_page, pool_slot, pool_head;
    long long slot_count;
    int B, rows, width, page_shift, heads, words;           // words: 16-byte words of one head's row
    int per_group;              // positions a workgroup copies
};

__global__ __launch_bounds__(256) void cache_commit_kernel(CommitArgs a)
{
    const int b = blockIdx.y, layer = blockIdx.z;
    int n = a.count ? a.count[b] : a.width;
    n = n < a.width ? n : a.width;
    const int j0 = blockIdx.x * a.per_group, j1 = min(n, j0 + a.per_group);
    const int row_words = a.heads * a.words;
    for (int i = threadIdx.x; i < (j1 - j0) * row_words; i += 256) {
        const int j = j0 + i / row_words, w = i % row_words;
        const int head = w / a.words, e = w % a.words;
        const long long slot = a.slots[(long long)b * a.width + j];
        const int r = a.row ? a.row[(long long)b * a.width + j] : j;
        if (slot < 0 || slot >= a.slot_count || r < 0 || r >= a.rows) continue;
        const long long src = layer * a.src_layer + b * a.src_batch + r * a.src_row + head * a.src_head + e;
        const long long dst = layer * a.pool_layer + (slot >> a.page_shift) * a.pool_page +
                              (slot & ((1ll << a.page_shift) - 1)) * a.pool_slot + head * a.pool_head + e;
        a.k_pool[dst] = a.k_rows[src];
        a.v_pool[dst] = a.v_rows[src];
    }
}

// ---- block tables, slot maps, free pages ---------------------------------------------------------------------------------
// The free pages are the entries taken .. given - 1 (modulo `pages`) of a ring; mark = {taken, given} only grows.  Demands are
// served in the order of the trajectories, from the ring's front as it was before the call; pages that are given back go to
// its end.  So one exclusive prefix sum over the demands and one over the returns say where every page goes.
struct PagesArgs {
    int32_t *table, *ring;
    const int32_t *length, *held, *add, *room;
    const long long *mark;
    int32_t *length_out, *held_out, *missing;
    long long *mark_out, *slots;
    int B, width, pages, page_shift, slot_width, default_room;
};

constexpr int kPagesThreads = 1024;

__global__ __launch_bounds__(kPagesThreads) void cache_pages_kernel(PagesArgs a)
{
    __shared__ long long sum_ask[kPagesThreads], sum_give[kPagesThreads];
    __shared__ long long base_ask, base_give, granted;
    const int t = threadIdx.x;
    const long long taken = a.mark[0], given = a.mark[1];
    long long avail = given - taken;
    avail = avail < 0 ? 0 : (avail > a.pages ? a.pages : avail);
    if (t == 0) { base_ask = 0; base_give = 0; granted = 0; }
    const long long ps = 1ll << a.page_shift;
    for (int b0 = 0; b0 < a.B; b0 += kPagesThreads) {
        const int b = b0 + t;
        long long len = 0, need = 0, ask = 0, give = 0;
        int held = 0, room = -1;
        if (b < a.B) {
            held = a.held[b];
            held = held < 0 ? 0 : (held > a.width ? a.width : held);
            room = a.room ? a.room[b] : a.default_room;
            if (room >= 0) {
                len = (long long)a.length[b] + (a.add ? a.add[b] : 0);
                len = len < 0 ? 0 : (len > held * ps ? held * ps : len);
                need = (len + room + ps - 1) >> a.page_shift;
            }
            ask = need > held && need <= a.width ? need - held : 0;
            give = held > need ? held - need : 0;
        }
        sum_ask[t] = ask; sum_give[t] = give;
        __syncthreads();
        for (int off = 1; off < kPagesThreads; off <<= 1) {
            const long long x = t >= off ? sum_ask[t - off] : 0, y = t >= off ? sum_give[t - off] : 0;
            __syncthreads();
            sum_ask[t] += x; sum_give[t] += y;
            __syncthreads();
        }
        if (b < a.B) {
            const long long before = base_ask + sum_ask[t] - ask, back = base_give + sum_give[t] - give;
            const bool ok = need <= held || (need <= a.width && before + ask <= avail);
            const int now = ok ? (int)need : held;
            int32_t *row = a.table + (long long)b * a.width;
            if (ok)
                for (long long i = 0; i < ask; ++i) row[held + i] = a.ring[(unsigned long long)(taken + before + i) % (unsigned)a.pages];
            for (long long i = 0; i < give; ++i) a.ring[(unsigned long long)(given + back + i) % (unsigned)a.pages] = row[need + i];
            a.length_out[b] = (int)len;
            a.held_out[b] = now;
            a.missing[b] = ok ? 0 : (int)(need - held);
            for (int j = 0; j < a.slot_width; ++j) {
                const long long pos = len + j, pg = pos >> a.page_shift;
                a.slots[(long long)b * a.slot_width + j] = j < room && pg < now ? (long long)row[pg] * ps + (pos & (ps - 1)) : -1;
            }
            if (ok && ask) atomicMax((unsigned long long *)&granted, (unsigned long long)(before + ask));
        }
        __syncthreads();
        if (t == 0) { base_ask += sum_ask[kPagesThreads - 1]; base_give += sum_give[kPagesThreads - 1]; }
        __syncthreads();
    }
    if (t == 0) { a.mark_out[0] = taken + granted; a.mark_out[1] = given + base_give; }
}

}  // namespace stand
