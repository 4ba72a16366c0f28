// serve_api.hip -- host side of the operators around a verification (include/stand.h): argument checks and launches.
// Nothing here allocates, waits or keeps state between calls; everything a call needs comes with it.
#include "cache_four.hpp"
#include "cache_ops.hpp"
#include "row_turns.hpp"
#include "serve_checks.hpp"
#include "serve_view.hpp"
#include "shape_logits.hpp"
#include "tree_attn.hpp"
#include "tree_attn4.hpp"

#include <algorithm>
#include <atomic>

using namespace stand;

namespace {

// The handle's device is current inside a call and the caller's is again after it.
struct DeviceScope {
    int before = -1;
    hipError_t e;
    explicit DeviceScope(int device)
    {
        e = hipGetDevice(&before);
        if (e == hipSuccess && before != device) e = hipSetDevice(device);
        else before = -1;
    }
    ~DeviceScope()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

int launched(const ServeView &v)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return STAND_OK;
    *v.last_hip = (int)e;
    return STAND_EHIP;
}

int bad_device(const ServeView &v, hipError_t e)
{
    *v.last_hip = (int)e;
    return STAND_EHIP;
}

// The form of the attention kernel a call takes, by the rows that share a key/value head, as if all nodes were drafted.
//   up to 32: four waves on different keys, each loading its own without a barrier (32 trees of 17 .. 32 rows, d 64: 44 us, with
//     tiles of 256 rows 51; up to 64 rows it would be behind: 90 us instead of 74, d 128);
//   up to 64: two waves of rows on each half of a stage's keys (32 trees, d 128: 72 us, with tiles of 256 rows 75; d 64: 42 and
//     49 us).  With d 128 it has 16 vector registers too few: they are stored and loaded again once per item, outside the loop;
//   above: eight waves of rows with d 128, 256 of them (four waves of rows on halves of the keys took the same times, 85 .. 89 us,
//     with 128 rows); with d 64 four, whose two workgroups share a compute unit (128 trees of 128 nodes: 190 us, eight: 207).
enum AttnForm { kAttn32, kAttn64, kAttnMore };
AttnForm attn_form(int64_t rows) { return rows <= 32 ? kAttn32 : rows <= 64 ? kAttn64 : kAttnMore; }

template <int D, bool F16, typename Call>
auto with_attn_shape(AttnForm f, Call call)
{
    switch (f) {
    case kAttn32: return call(AttnShape<D, F16, 1, 4, 1>{});
    case kAttn64: return call(AttnShape<D, F16, 2, 2, 1>{});
    default: return call(AttnShape<D, F16, D == 64 ? 4 : 8, 1, 2>{});
    }
}
// Over a cache of 4 bits: up to 64 rows a wave for each 32, more than that four waves of rows with the same keys.  Between 33 and 64 rows
// either may be ahead, as many trajectories or one: four heads of keys, d 128, all nodes drafted, waves by themselves and teams, us:
//     rows          36           48           56           64
//     1000 .. 9000 tokens, 32 trees     43, 55       48, 58       53, 57       54, 59       (three quarters drafted, 64 rows: 49, 57)
//     200 .. 3000, 128 trees, 8 heads   110, 141     145, 146     157, 146     163, 148
//     60 000, one tree                  55, 40       56, 40       57, 40       59, 41
//     40, one tree                      15, 16       15, 16       15, 16       15, 17
// and d 64 likewise (32 trees 31, 40 .. 37, 43; 128 trees 77, 95 .. 119, 98; one long 44, 32 .. 47, 33; one short 14, 12).  Lengths are the GPU's
// alone, so the rule is by rows, and for batches, of whose trees a part is not drafted.
template <int D, bool F16, typename Call>
auto with_attn4_shape(AttnForm f, Call call)
{
    return f == kAttnMore ? call(Attn4Shape<D, F16, 4>{}) : call(Attn4Shape<D, F16, 1>{});
}
template <typename Call>
auto with_attn_shape(const stand_cache *c, AttnForm f, Call call)
{
    const bool f16 = rows_dtype(c) == STAND_F16;
    if (of_four(c)) {
        if (c->head_dim == 64) return f16 ? with_attn4_shape<64, true>(f, call) : with_attn4_shape<64, false>(f, call);
        return f16 ? with_attn4_shape<128, true>(f, call) : with_attn4_shape<128, false>(f, call);
    }
    if (c->head_dim == 64) return f16 ? with_attn_shape<64, true>(f, call) : with_attn_shape<64, false>(f, call);
    return f16 ? with_attn_shape<128, true>(f, call) : with_attn_shape<128, false>(f, call);
}
template <int D, bool F16, int WR, int WK, int SUB>
const void *kernel_of(AttnShape<D, F16, WR, WK, SUB>) { return (const void *)tree_attn_kernel<AttnShape<D, F16, WR, WK, SUB>>; }
template <int D, bool F16, int WR>
const void *kernel_of(Attn4Shape<D, F16, WR>) { return (const void *)tree_attn4_kernel<Attn4Shape<D, F16, WR>>; }
template <int D, bool F16, int WR, int WK, int SUB>
void run_kernel(AttnShape<D, F16, WR, WK, SUB>, dim3 grid, dim3 threads, const TreeAttnArgs &a, hipStream_t s)
{
    using S = AttnShape<D, F16, WR, WK, SUB>;
    tree_attn_kernel<S><<<grid, threads, S::BYTES, s>>>(a);
}
template <int D, bool F16, int WR>
void run_kernel(Attn4Shape<D, F16, WR>, dim3 grid, dim3 threads, const TreeAttn4Args &a, hipStream_t s)
{
    using S = Attn4Shape<D, F16, WR>;
    tree_attn4_kernel<S><<<grid, threads, S::BYTES, s>>>(a);
}
// Shares of a launch of that many workgroups.
template <int D, bool F16, int WR, int WK, int SUB>
int shares_of(AttnShape<D, F16, WR, WK, SUB>, int workgroups) { return workgroups; }
template <int D, bool F16, int WR>
int shares_of(Attn4Shape<D, F16, WR>, int workgroups) { return workgroups * Attn4Shape<D, F16, WR>::TEAMS; }

// The cache as kernels that count in 16-byte chunks see it.
CachePlaces places_of(const stand_cache *c)
{
    CachePlaces p;
    const int64_t chunk = of_four(c) ? 32 : 8;
    p.k = (char *)c->d_k; p.v = (char *)c->d_v;
    p.layer = c->layer_stride / chunk; p.page = c->page_stride / chunk; p.slot = c->slot_stride / chunk; p.head = c->head_stride / chunk;
    p.k_scale = p.v_scale = nullptr;
    p.scale_layer = p.scale_page = p.scale_slot = p.scale_head = 0;
    if (of_four(c)) {
        const stand_cache4 *f = four_of(c);
        p.k_scale = (uint8_t *)f->d_k_scale; p.v_scale = (uint8_t *)f->d_v_scale;
        p.scale_layer = f->scale_layer_stride; p.scale_page = f->scale_page_stride; p.scale_slot = f->scale_slot_stride;
        p.scale_head = f->scale_head_stride;
    }
    p.page_shift = log2_of(c->page_size); p.pages = c->pages;
    return p;
}

// The kernel's view of the rows of stand_tree_rotate and stand_cache_append; -> workgroups of a trajectory.
unsigned turn_args(TurnArgs &a, int64_t B, const stand_rotation *rotation, const stand_turned_rows *rows, bool values)
{
    a.q = (const uint16_t *)rows->d_q; a.k = (const uint16_t *)rows->d_k; a.v = (const uint16_t *)rows->d_v;
    a.q_out = (uint16_t *)rows->d_q_out; a.k_out = (uint16_t *)rows->d_k_out;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = rows->q_stride[i]; a.ks[i] = rows->k_stride[i]; a.vs[i] = rows->v_stride[i];
        a.qos[i] = rows->q_out_stride[i]; a.kos[i] = rows->k_out_stride[i];
    }
    a.turns = nullptr; a.q_norm = a.k_norm = nullptr; a.eps = 0.0; a.positions = a.half = 0;
    if (rotation) {
        a.turns = rotation->d_turns; a.positions = rotation->positions; a.half = rotation->dims / 2;
        a.q_norm = (const uint16_t *)rotation->d_q_norm; a.k_norm = (const uint16_t *)rotation->d_k_norm; a.eps = rotation->eps;
    }
    a.rows = rows->rows; a.q_heads = a.q ? rows->q_heads : 0; a.kv_heads = rows->kv_heads;
    // A thread has up to four heads of its row, whose cosines and weights it makes once (128 trees of 128, 16/8 heads of 128: 27 us, two heads 30,
    // one 37; as many heads as leave a wave one row 35); where one head would not make 1024 workgroups, one.
    const int many = B * turn_groups(rows->rows, a.q_heads + 2ll * a.kv_heads, rows->head_dim) >= 1024 ? 4 : 1;
    a.q_step = (a.q_heads + many - 1) / many;
    a.k_step = (a.kv_heads + many - 1) / many;
    a.q_groups = a.q ? (int)turn_groups(rows->rows, a.q_step, rows->head_dim) : 0;
    a.k_groups = (int)turn_groups(rows->rows, a.k_step, rows->head_dim);
    a.tok = nullptr; a.anc = nullptr; a.anc_words = 0; a.start = a.count = nullptr;
    a.slots = nullptr; a.width = 0; a.slot_count = 0;
    return (unsigned)(a.q_groups + (values ? 2 : 1) * a.k_groups);
}
template <TurnTarget TO, bool NEIGHBOURS>
void turn_launch(const TurnArgs &a, const stand_turned_rows *rows, dim3 grid, hipStream_t s)
{
    const dim3 threads(kTurnThreads);
    const bool f16 = rows->dtype == STAND_F16;
    static_assert(turn_heads_of_group(64) == 64 && turn_heads_of_group(128) == 32, "turn_groups() counts with these");
    if (rows->head_dim == 64) {
        if (f16) row_turns_kernel<64, true, TO, NEIGHBOURS><<<grid, threads, 0, s>>>(a);
        else row_turns_kernel<64, false, TO, NEIGHBOURS><<<grid, threads, 0, s>>>(a);
    } else {
        if (f16) row_turns_kernel<128, true, TO, NEIGHBOURS><<<grid, threads, 0, s>>>(a);
        else row_turns_kernel<128, false, TO, NEIGHBOURS><<<grid, threads, 0, s>>>(a);
    }
}
template <TurnTarget TO>
void turn_launch(const TurnArgs &a, const stand_rotation *rotation, const stand_turned_rows *rows, unsigned groups, int B, hipStream_t s)
{
    const dim3 grid(groups, (unsigned)B);
    if (rotation && rotation->neighbours) turn_launch<TO, true>(a, rows, grid, s);
    else turn_launch<TO, false>(a, rows, grid, s);
}

// Workgroups of a launch: as many as the device holds at once, a multiple of its eight XCDs; 0: the device refused.  (Above
// 64 KiB dynamic LDS has to be asked for, on every device.)
constexpr int kMaxDevices = 64;
template <typename S>
int attn_groups_of(const ServeView &v)
{
    static_assert(S::BYTES <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<int> known[kMaxDevices];
    const int at = v.device < kMaxDevices ? v.device : -1;
    int per_cu = at < 0 ? 0 : known[at].load(std::memory_order_relaxed);
    if (per_cu == 0) {
        const DeviceScope scope(v.device);
        const void *kernel = kernel_of(S{});
        hipError_t e = scope.e;
        if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::BYTES);
        if (e == hipSuccess) e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, S::THREADS, S::BYTES);
        if (e != hipSuccess || per_cu < 1) {
            *v.last_hip = (int)e;
            return 0;
        }
        if (at >= 0) known[at].store(per_cu, std::memory_order_relaxed);
    }
    return std::max(8, v.cus * per_cu / 8 * 8);
}
// Workspace: records, places, parts.
template <typename S>
uint64_t attn_work_bytes(int groups)
{
    return (uint64_t)groups * (sizeof(JoinRecord) + S::TM * 8 + 2 * S::TM * (S::D + 2) * 4);
}

template <typename S>
hipError_t attn_launch(TreeAttn4Args &a, hipStream_t s)
{
    a.groups = shares_of(S{}, a.workgroups);
    a.place = (long long *)(a.join + a.groups);
    a.part = (float *)(a.place + (size_t)a.groups * S::TM);
    const dim3 grid((unsigned)a.workgroups), threads(S::THREADS);
    run_kernel(S{}, grid, threads, a, s);
    tree_attn_join_kernel<S::D, S::TM, S::F16><<<dim3((unsigned)a.groups, S::WR), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

extern "C" uint64_t stand_tree_attention_work(const stand_handle *h, const stand_cache *cache, int32_t q_heads)
{
    if (!h) return 0;
    const ServeView v = serve_view(const_cast<stand_handle *>(h));
    if (check_attention_size(v.B, cache, q_heads) != STAND_OK) return 0;
    const AttnForm f = attn_form((int64_t)v.N * (q_heads / cache->kv_heads));
    return with_attn_shape(cache, f,
                           [&](auto s) { return attn_work_bytes<decltype(s)>(shares_of(s, attn_groups_of<decltype(s)>(v))); });
}

extern "C" int stand_tree_attention(stand_handle *h, const stand_cache *cache, int32_t layer, const int32_t *d_len,
                                    const int32_t *d_table, int32_t table_width, const int32_t *d_draft_tok,
                                    const stand_tree_rows *rows, void *d_work, uint64_t work_bytes, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_tree_attention(v.B, cache, layer, d_len, d_table, table_width, d_draft_tok, rows, d_work);
    if (refused) return refused;
    TreeAttn4Args a;
    a.q = (const uint16_t *)rows->d_q; a.k_new = (const uint16_t *)rows->d_k; a.v_new = (const uint16_t *)rows->d_v;
    a.out = (uint16_t *)rows->d_out;
    const bool four = of_four(cache);
    a.k_pool = (const uint16_t *)cache->d_k + layer * cache->layer_stride / (four ? 4 : 1);
    a.v_pool = (const uint16_t *)cache->d_v + layer * cache->layer_stride / (four ? 4 : 1);
    a.k_scale = a.v_scale = nullptr;
    a.scale_page = a.scale_slot = a.scale_head = 0;
    if (four) {
        const stand_cache4 *f = four_of(cache);
        a.k_scale = (const uint8_t *)f->d_k_scale + layer * f->scale_layer_stride;
        a.v_scale = (const uint8_t *)f->d_v_scale + layer * f->scale_layer_stride;
        a.scale_page = f->scale_page_stride; a.scale_slot = f->scale_slot_stride; a.scale_head = f->scale_head_stride;
    }
    a.len = d_len; a.table = d_table; a.draft_tok = d_draft_tok;
    a.anc = (const uint32_t *)v.anc; a.anc_words = 2 * v.anc_words;      // (little endian: words of 32 nodes)
    a.join = (JoinRecord *)d_work;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = rows->q_stride[i]; a.ks[i] = rows->k_stride[i]; a.vs[i] = rows->v_stride[i]; a.os[i] = rows->out_stride[i];
    }
    a.pool_page = cache->page_stride; a.pool_slot = cache->slot_stride; a.pool_head = cache->head_stride;
    a.scale = rows->scale; a.B = v.B; a.N = v.N; a.kv_heads = cache->kv_heads; a.per_kv = rows->q_heads / cache->kv_heads;
    a.width = table_width; a.pages = cache->pages; a.page_shift = log2_of(cache->page_size);
    return with_attn_shape(cache, attn_form((int64_t)v.N * a.per_kv), [&](auto s) {
        using S = decltype(s);
        a.workgroups = attn_groups_of<S>(v);
        if (a.workgroups == 0) return STAND_EHIP;
        if (work_bytes < attn_work_bytes<S>(shares_of(s, a.workgroups))) return STAND_EINVAL;
        const DeviceScope scope(v.device);
        if (scope.e != hipSuccess) return bad_device(v, scope.e);
        const hipError_t e = attn_launch<S>(a, (hipStream_t)stream);
        return e == hipSuccess ? STAND_OK : bad_device(v, e);
    });
}

extern "C" int stand_cache_commit(stand_handle *h, const stand_cache *cache, const stand_cache_rows *rows, const int64_t *d_slots,
                                  int32_t width, const int32_t *d_row, const int32_t *d_count, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_cache_commit(v.B, cache, rows, d_slots, width);
    if (refused) return refused;
    if (of_four(cache)) {
        CommitFourArgs a;
        a.units = cache->head_dim / kFourUnit;
        a.heads = cache->kv_heads;
        a.per_group = four_per_group(a.heads * a.units);
        const int64_t groups = commit_groups(width, a.per_group);
        const DeviceScope scope(v.device);
        if (scope.e != hipSuccess) return bad_device(v, scope.e);
        a.k_rows = (const uint4 *)rows->d_k; a.v_rows = (const uint4 *)rows->d_v;
        a.to = places_of(cache);
        a.slots = d_slots; a.row = d_row; a.count = d_count;
        a.src_layer = rows->layer_stride / 8; a.src_batch = rows->batch_stride / 8; a.src_row = rows->row_stride / 8; a.src_head = rows->head_stride / 8;
        a.slot_count = (long long)cache->pages << a.to.page_shift;
        a.rows = rows->rows; a.width = width;
        const dim3 grid((unsigned)groups, (unsigned)v.B, (unsigned)cache->layers), threads(kCommitThreads);
        if (rows_dtype(cache) == STAND_F16) cache_commit4_kernel<true><<<grid, threads, 0, (hipStream_t)stream>>>(a);
        else cache_commit4_kernel<false><<<grid, threads, 0, (hipStream_t)stream>>>(a);
        return launched(v);
    }
    CommitArgs a;
    a.words = cache->head_dim / 8;
    a.heads = cache->kv_heads;
    a.per_group = commit_per_group(a.heads * a.words);
    const int64_t groups = commit_groups(width, a.per_group);
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    a.k_rows = (const uint4 *)rows->d_k; a.v_rows = (const uint4 *)rows->d_v;
    a.k_pool = (uint4 *)cache->d_k; a.v_pool = (uint4 *)cache->d_v;
    a.slots = d_slots; a.row = d_row; a.count = d_count;
    a.src_layer = rows->layer_stride / 8; a.src_batch = rows->batch_stride / 8; a.src_row = rows->row_stride / 8; a.src_head = rows->head_stride / 8;
    a.pool_layer = cache->layer_stride / 8; a.pool_page = cache->page_stride / 8; a.pool_slot = cache->slot_stride / 8;
    a.pool_head = cache->head_stride / 8;
    a.page_shift = log2_of(cache->page_size);
    a.slot_count = (long long)cache->pages << a.page_shift;
    a.B = v.B; a.rows = rows->rows; a.width = width;
    cache_commit_kernel<<<dim3((unsigned)groups, (unsigned)v.B, (unsigned)cache->layers), dim3(kCommitThreads), 0, (hipStream_t)stream>>>(a);
    return launched(v);
}

extern "C" int stand_cache_read(stand_handle *h, const stand_cache *cache, int32_t first_layer, int32_t layers, const int32_t *d_table,
                                int32_t table_width, const int32_t *d_start, const int32_t *d_count, const stand_cache_rows_out *rows, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_cache_read(v.B, cache, first_layer, layers, d_table, table_width, rows);
    if (refused) return refused;
    ReadArgs a;
    a.units = cache->head_dim / kReadUnit;
    a.heads = cache->kv_heads;
    a.per_group = four_per_group(a.heads * a.units);
    const int64_t groups = commit_groups(rows->rows, a.per_group);
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    a.k_rows = (uint4 *)rows->d_k; a.v_rows = (uint4 *)rows->d_v;
    a.from = places_of(cache);
    a.table = d_table; a.start = d_start; a.count = d_count;
    a.dst_layer = rows->layer_stride / 8; a.dst_batch = rows->batch_stride / 8; a.dst_row = rows->row_stride / 8; a.dst_head = rows->head_stride / 8;
    a.first_layer = first_layer; a.rows = rows->rows; a.width = table_width;
    const dim3 grid((unsigned)groups, (unsigned)v.B, (unsigned)layers), threads(kCommitThreads);
    if (!of_four(cache)) cache_read_kernel<kRead16><<<grid, threads, 0, (hipStream_t)stream>>>(a);
    else if (rows_dtype(cache) == STAND_F16) cache_read_kernel<kReadF16><<<grid, threads, 0, (hipStream_t)stream>>>(a);
    else cache_read_kernel<kReadBf16><<<grid, threads, 0, (hipStream_t)stream>>>(a);
    return launched(v);
}

extern "C" int stand_tree_rotate(stand_handle *h, const stand_rotation *rotation, const int32_t *d_len, const int32_t *d_draft_tok,
                                 const stand_turned_rows *rows, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_tree_rotate(v.B, v.N, rotation, d_len, d_draft_tok, rows);
    if (refused) return refused;
    TurnArgs a;
    const unsigned groups = turn_args(a, v.B, rotation, rows, false);
    a.start = d_len; a.tok = d_draft_tok; a.anc = v.anc; a.anc_words = v.anc_words;
    a.to = CachePlaces{};
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    // (what it takes and saves, alone and with its reader: put_row in row_turns.hpp; of a tree's rows a third to a half are not drafted)
    const bool past = (int64_t)v.B * rows->rows * (a.q_heads + (int64_t)a.kv_heads) * rows->head_dim * 2 > ((int64_t)64 << 20);
    if (past) turn_launch<kTurnRowsPast>(a, rotation, rows, groups, v.B, (hipStream_t)stream);
    else turn_launch<kTurnRows>(a, rotation, rows, groups, v.B, (hipStream_t)stream);
    return launched(v);
}

extern "C" int stand_cache_append(stand_handle *h, const stand_cache *cache, int32_t layer, const stand_rotation *rotation,
                                  const stand_turned_rows *rows, const int32_t *d_start, const int64_t *d_slots, int32_t width,
                                  const int32_t *d_count, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_cache_append(v.B, cache, layer, rotation, rows, d_slots, width);
    if (refused) return refused;
    TurnArgs a;
    const unsigned groups = turn_args(a, v.B, rotation, rows, true);
    a.start = d_start; a.count = d_count; a.slots = d_slots; a.width = width;
    a.to = places_of(cache);
    a.to.k += layer * a.to.layer * 16; a.to.v += layer * a.to.layer * 16;
    if (a.to.k_scale) { a.to.k_scale += layer * a.to.scale_layer; a.to.v_scale += layer * a.to.scale_layer; }
    a.slot_count = (long long)cache->pages << a.to.page_shift;
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    if (of_four(cache)) turn_launch<kTurnCache4>(a, rotation, rows, groups, v.B, (hipStream_t)stream);
    else turn_launch<kTurnCache16>(a, rotation, rows, groups, v.B, (hipStream_t)stream);
    return launched(v);
}

extern "C" int stand_cache_pages(stand_handle *h, const stand_pages *p, const int32_t *d_add, const int32_t *d_room, int64_t *d_slots,
                                 int32_t slot_width, int32_t *d_missing, const stand_pages *out, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_cache_pages(v.B, p, d_slots, slot_width, d_missing, out);
    if (refused) return refused;
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    PagesArgs a;
    a.table = p->d_table; a.ring = p->d_ring; a.length = p->d_length; a.held = p->d_held; a.add = d_add; a.room = d_room;
    a.mark = (const long long *)p->d_mark;
    a.length_out = out->d_length; a.held_out = out->d_held; a.missing = d_missing; a.mark_out = (long long *)out->d_mark;
    a.slots = (long long *)d_slots;
    a.B = v.B; a.width = p->width; a.pages = p->pages; a.page_shift = log2_of(p->page_size); a.slot_width = slot_width;
    a.default_room = v.D + 1;
    // One workgroup where that is little work (up to 64 trajectories with 4096 slots: the state is then written behind its own
    // reads); else one for each trajectory, up to 1024 of them.
    const bool aside = out->d_length != p->d_length && out->d_held != p->d_held && out->d_mark != p->d_mark;
    const int64_t slots = (int64_t)v.B * slot_width;
    static_assert(kServeMaxBatch <= kPagesMine * kPagesGroups, "a workgroup's trajectories stand in LDS");
    int64_t groups = v.B <= kPagesMine && slots <= 4096 ? 1 : std::min<int64_t>(v.B, kPagesGroups);
    a.per_group = (int)((v.B + groups - 1) / groups);
    groups = (v.B + a.per_group - 1) / a.per_group;
    a.what = groups == 1 || aside ? kPagesTables | kPagesState : kPagesTables;
    cache_pages_kernel<<<dim3((unsigned)groups), dim3(kPagesThreads), 0, (hipStream_t)stream>>>(a);
    if (!(a.what & kPagesState)) {
        a.what = kPagesState;
        cache_pages_kernel<<<dim3(1), dim3(kPagesThreads), 0, (hipStream_t)stream>>>(a);
    }
    return launched(v);
}

extern "C" uint64_t stand_shape_logits_work(const stand_handle *h)
{
    if (!h) return 0;
    const ServeView v = serve_view(const_cast<stand_handle *>(h));
    return (uint64_t)v.B * v.N;
}

extern "C" int stand_shape_logits(stand_handle *h, const void *d_logits, void *d_out, const int32_t *d_draft_tok, const int32_t *d_count,
                                  const float *d_penalty, const int32_t *d_bias_id, const float *d_bias, int32_t bias_width,
                                  const uint32_t *d_allow, void *d_work, uint64_t work_bytes, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_shape_logits(v.B, v.logits_dtype, d_logits, d_out, d_draft_tok, d_bias_id, d_bias, bias_width);
    if (refused) return refused;
    if (d_allow && (!d_work || work_bytes < stand_shape_logits_work(h))) return STAND_EINVAL;
    const bool f32 = v.logits_dtype == STAND_F32;
    ShapeArgs a;
    a.x = d_logits; a.out = d_out; a.draft_tok = d_draft_tok; a.count = d_count; a.penalty = d_penalty; a.bias_id = d_bias_id; a.bias = d_bias;
    a.allow = d_allow; a.anc = v.anc; a.anc_words = v.anc_words; a.N = v.N; a.V = v.V; a.M = bias_width; a.words = (v.V + 31) / 32;
    a.any = (uint8_t *)d_work; a.rows = (long long)v.B * v.N;
    const int64_t spans = ((int64_t)v.V + kShapeSpan - 1) / kShapeSpan;
    // nodes that share a workgroup's counts: as many as leave 2048 workgroups, at most 16
    a.nodes_per_group = kShapeNodes;
    while (a.nodes_per_group > 1 && spans * v.B * ((v.N + a.nodes_per_group - 1) / a.nodes_per_group) < 2048) a.nodes_per_group /= 2;
    a.node_groups = (v.N + a.nodes_per_group - 1) / a.nodes_per_group;
    a.spans = (int)spans;
    if (spans * a.node_groups * v.B > (int64_t)(UINT32_MAX / kShapeThreads)) return STAND_ELIMIT;
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    const dim3 grid((unsigned)(spans * a.node_groups * v.B));
    if (d_allow) shape_rows_kernel<<<dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, (hipStream_t)stream>>>(a);
    if (f32) shape_logits_kernel<kDtF32><<<grid, dim3(kShapeThreads), 0, (hipStream_t)stream>>>(a);
    else shape_logits_kernel<kDtBf16><<<grid, dim3(kShapeThreads), 0, (hipStream_t)stream>>>(a);
    return launched(v);
}

extern "C" int stand_count_tokens(stand_handle *h, int32_t *d_count, const int32_t *d_tok, const int32_t *d_len, int32_t width,
                                  int32_t prompt, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_count_tokens(v.B, d_count, d_tok, width);
    if (refused) return refused;
    const int64_t groups = ((int64_t)width + 255) / 256;
    const DeviceScope scope(v.device);
    if (scope.e != hipSuccess) return bad_device(v, scope.e);
    count_tokens_kernel<<<dim3((unsigned)groups, (unsigned)v.B), dim3(256), 0, (hipStream_t)stream>>>(d_count, d_tok, d_len, v.V, width, prompt);
    return launched(v);
}
