// cache_ops.hpp -- the paged key/value cache between two target model passes: rows into their slots, and the pages of
// each trajectory (block tables, slot maps, the ring of free pages).  Everything these kernels decide by is on the device
// (accepted lengths, accepted nodes), so that a serving loop never waits for the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "commit_plan.hpp"

namespace stand {

// ---- rows into the cache ------------------------------------------------------------------------------------------------
// For every layer, trajectory b and j < count[b]: the keys and values of source row row[b][j] go to slot slots[b][j].  A slot
// is page * page_size + place in the page.  All strides are in 16-byte words.  A thread copies 16 bytes of a key, then of a value,
// then the next pair: four to eight of them where there are as many positions, more where a row has more than 1024 words.  Bound by HBM
// with prompts (751 MB in and out, 16 layers x 4 x 2100 rows of 2 KB: 148 us, 5.1 TB/s).  After a step it is bound by its trips to
// memory, one behind the other: count, then slot, key and value for each pair, two or three times (5.5 us for 28 layers of 32 short
// paths); the pairs do not depend on each other, but the compiler may not load past a store.
struct CommitArgs {
    const uint4 *k_rows, *v_rows;
    uint4 *k_pool, *v_pool;
    const int64_t *slots;       // [B][width]
    const int32_t *row, *count; // [B][width] or NULL (row j), [B] or NULL (width)
    long long src_layer, src_batch, src_row, src_head;      // keys' and values' rows have the same strides
    long long pool_layer, pool_page, pool_slot, pool_head;
    long long slot_count;
    int B, rows, width, page_shift, heads, words;           // words: 16-byte words of one head's row
    int per_group;              // positions a workgroup copies at a time
};

__global__ __launch_bounds__(kCommitThreads) void cache_commit_kernel(CommitArgs a)
{
    const int b = blockIdx.y, layer = blockIdx.z;
    const int n = commit_positions(a.count ? a.count[b] : a.width, a.width);
    const int row_words = a.heads * a.words;
    for (unsigned j0 = blockIdx.x * (unsigned)a.per_group; j0 < (unsigned)n; j0 += gridDim.x * (unsigned)a.per_group) {
        const int words = commit_words(n, j0, a.per_group, row_words);
        for (int i = threadIdx.x; i < words; i += kCommitThreads) {
            const int j = (int)j0 + i / row_words, w = i % row_words;
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
}

// ---- block tables, slot maps, free pages ---------------------------------------------------------------------------------
// The free pages are the entries taken .. given - 1 (modulo `pages`) of a ring; mark = {taken, given} only grows.  Demands are
// served in the order of the trajectories, from the ring's front as it was before the call; pages that are given back go to
// its end.  So one exclusive prefix sum over the demands and one over the returns say where every page goes, and every
// workgroup can make those sums for itself: `groups` of them share the trajectories' tables and slots, none waits for another.
// What is taken and what is given back are different entries of the ring, and a slot on a new page is read from the ring, not
// from the table.  The new lengths, held counts and marks may replace the old ones, which the others still read: then they are
// written by a launch of their own behind the others' (`what`), or, where there is one workgroup only, after a barrier.
// Bound by latency: marks and demands, sums, pages, state.  32 trajectories after a step take 5.9 us, 512 with up to 4000 slots
// each (16 MB) 10.4 us.  (All threads on one trajectory after the other: 9.6 and 16.7 us.)
struct PagesArgs {
    int32_t *table, *ring;
    const int32_t *length, *held, *add, *room;
    const long long *mark;
    int32_t *length_out, *held_out, *missing;
    long long *mark_out, *slots;
    int B, width, pages, page_shift, slot_width, default_room;
    int per_group;              // consecutive trajectories of a workgroup, at most kPagesMine
    int what;                   // kPagesTables | kPagesState
};
constexpr int kPagesTables = 1, kPagesState = 2;
constexpr int kPagesThreads = 512;   // (256: 11.6 us for 512 trajectories with 4000 slots each, 1024: 14.8, this: 10.5)
constexpr int kPagesMine = 64;       // trajectories of a workgroup: 1024 of them have all
constexpr int kPagesGroups = 1024;
constexpr int kPagesKept = 2;        // of a thread's trajectories, in registers
constexpr int kPagesFirst = 8;       // a step takes one page or two of a trajectory

struct PagesDemand { long long len; int need, held, ask, give, room; };

__device__ __forceinline__ PagesDemand pages_demand(const PagesArgs &a, int b)
{
    PagesDemand d;
    const long long ps = 1ll << a.page_shift;
    d.held = a.held[b];
    d.held = d.held < 0 ? 0 : (d.held > a.width ? a.width : d.held);
    d.room = a.room ? a.room[b] : a.default_room;
    d.len = 0;
    long long need = 0;
    if (d.room >= 0) {
        d.len = (long long)a.length[b] + (a.add ? a.add[b] : 0);
        d.len = d.len < 0 ? 0 : (d.len > d.held * ps ? d.held * ps : d.len);
        need = (d.len + d.room + ps - 1) >> a.page_shift;
    }
    need = need < 0x7FFFFFFF ? need : 0x7FFFFFFF;
    d.need = (int)need;
    d.ask = need > d.held && need <= a.width ? (int)need - d.held : 0;
    d.give = d.held > need ? d.held - (int)need : 0;
    return d;
}

__global__ __launch_bounds__(kPagesThreads) void cache_pages_kernel(PagesArgs a)
{
    struct Mine { long long len, before, back; int need, held, now, ask, give, room; };
    __shared__ Mine mine[kPagesMine];
    __shared__ long long wave_ask[kPagesThreads / 64], wave_give[kPagesThreads / 64];
    __shared__ unsigned long long granted;
    __shared__ int most;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const long long taken = a.mark[0], given = a.mark[1];
    long long avail = given - taken;
    avail = avail < 0 ? 0 : (avail > a.pages ? a.pages : avail);
    const int chunk = (a.B + kPagesThreads - 1) / kPagesThreads, c0 = t * chunk, c1 = min(a.B, c0 + chunk);
    const int b0 = blockIdx.x * a.per_group, b1 = min(a.B, b0 + a.per_group);

    // sums before this thread's trajectories; what the first ones ask for is kept
    long long ask = 0, give = 0;
    PagesDemand kept[kPagesKept];
#pragma unroll
    for (int q = 0; q < kPagesKept; ++q) kept[q] = pages_demand(a, min(c0 + q, a.B - 1));
#pragma unroll
    for (int q = 0; q < kPagesKept; ++q)
        if (c0 + q < c1) { ask += kept[q].ask; give += kept[q].give; }
    for (int b = c0 + kPagesKept; b < c1; ++b) {
        const PagesDemand d = pages_demand(a, b);
        ask += d.ask; give += d.give;
    }
    long long up_ask = ask, up_give = give;
    for (int off = 1; off < 64; off <<= 1) {
        const long long x = __shfl_up(up_ask, off), y = __shfl_up(up_give, off);
        if (lane >= off) { up_ask += x; up_give += y; }
    }
    if (lane == 63) { wave_ask[wave] = up_ask; wave_give[wave] = up_give; }
    if (t == 0) { granted = 0; most = 0; }
    __syncthreads();
    long long before = up_ask - ask, back = up_give - give;
    for (int k = 0; k < wave; ++k) { before += wave_ask[k]; back += wave_give[k]; }

    // what becomes of each
    const bool state = a.what & kPagesState;
    long long all_given = 0;
    for (int k = 0; k < kPagesThreads / 64; ++k) all_given += wave_give[k];
    auto settle = [&](int b, const PagesDemand &d) {
        const bool ours = b >= b0 && b < b1;
        const bool ok = d.need <= d.held || (d.need <= a.width && before + d.ask <= avail);
        const int now = ok ? d.need : d.held;
        if (state && blockIdx.x == 0 && ok && d.ask) atomicMax(&granted, (unsigned long long)(before + d.ask));
        if (ours && (a.what & kPagesTables)) {
            a.missing[b] = ok ? 0 : d.need - d.held;
            mine[b - b0] = Mine{d.len, before, back, d.need, d.held, now, ok ? d.ask : 0, d.give, d.room};
            if (ok && d.ask + d.give > kPagesFirst) atomicMax(&most, d.ask + d.give);
        }
        if (state && !(a.what & kPagesTables)) { a.length_out[b] = (int)d.len; a.held_out[b] = now; }
        before += d.ask; back += d.give;
    };
#pragma unroll
    for (int q = 0; q < kPagesKept; ++q)
        if (c0 + q < c1) settle(c0 + q, kept[q]);
    for (int b = c0 + kPagesKept; b < c1; ++b) settle(b, pages_demand(a, b));
    __syncthreads();
    if (state && t == 0 && blockIdx.x == 0) { a.mark_out[0] = taken + (long long)granted; a.mark_out[1] = given + all_given; }
    if (!(a.what & kPagesTables)) return;

    const long long ps = 1ll << a.page_shift;
    const unsigned P = (unsigned)a.pages, taken_at = (unsigned)((unsigned long long)taken % P), given_at = (unsigned)((unsigned long long)given % P);
    auto ring_at = [&](unsigned start, long long i) {          // (i < pages where the ring is whole)
        const unsigned long long x = (unsigned long long)start + (unsigned long long)i;
        return (unsigned)(x < P ? x : x - P < P ? x - P : x % P);
    };
    const int n = b1 - b0;
    // A trajectory either takes pages or gives some back: from one place in the ring or the table to one in the other.
    auto from = [&](int k, const Mine &m, int i) {
        return m.ask ? a.ring + ring_at(taken_at, m.before + i) : a.table + (long long)(b0 + k) * a.width + m.need + i;
    };
    auto to = [&](int k, const Mine &m, int i) {
        return m.ask ? a.table + (long long)(b0 + k) * a.width + m.held + i : a.ring + ring_at(given_at, m.back + i);
    };
    // the first few of all trajectories at once, a thread each; the rest of those that move many by teams of threads
    for (int x = t; x < n * kPagesFirst; x += kPagesThreads) {
        const int k = x / kPagesFirst, i = x % kPagesFirst;
        const Mine &m = mine[k];
        if (i < m.ask + m.give) *to(k, m, i) = *from(k, m, i);
    }
    int team = kPagesThreads;
    while (team > 64 && team * n > kPagesThreads) team /= 2;
    const int at = t & (team - 1);
    if (most)
        for (int k = t / team; k < n; k += kPagesThreads / team) {
            const Mine &m = mine[k];
            const int count = m.ask + m.give;
            for (int i0 = kPagesFirst + at; i0 < count; i0 += 4 * team) {
                int32_t page[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) page[u] = i0 + u * team < count ? *from(k, m, i0 + u * team) : 0;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i0 + u * team < count) *to(k, m, i0 + u * team) = page[u];
            }
        }
    auto slot_of = [&](int k, int j) {
        const Mine &m = mine[k];
        const long long pos = m.len + j, pg = pos >> a.page_shift;
        if (j >= m.room || pg >= m.now) return -1ll;
        const int page = pg < m.held ? a.table[(long long)(b0 + k) * a.width + pg] : a.ring[ring_at(taken_at, m.before + pg - m.held)];
        return (long long)page * ps + (pos & (ps - 1));
    };
    long long *slots = a.slots + (long long)b0 * a.slot_width;
    if (a.slot_width < 64)
        for (int x = t; x < n * a.slot_width; x += kPagesThreads) slots[x] = slot_of(x / a.slot_width, x % a.slot_width);
    else
        for (int k = t / team; k < n; k += kPagesThreads / team)
            for (int j0 = at; j0 < a.slot_width; j0 += 4 * team) {
                long long slot[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) slot[u] = j0 + u * team < a.slot_width ? slot_of(k, j0 + u * team) : 0;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (j0 + u * team < a.slot_width) slots[(long long)k * a.slot_width + j0 + u * team] = slot[u];
            }
    if (state)
        for (int k = t; k < n; k += kPagesThreads) { a.length_out[b0 + k] = (int)mine[k].len; a.held_out[b0 + k] = mine[k].now; }
}

}  // namespace stand
