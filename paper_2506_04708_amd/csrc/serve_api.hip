// serve_api.hip -- host side of the operators around a verification (include/stand.h): argument checks and launches.
// Nothing here allocates, waits or keeps state between calls; everything a call needs comes with it.
#include "cache_ops.hpp"
#include "serve_checks.hpp"
#include "serve_view.hpp"
#include "shape_logits.hpp"
#include "tree_attn.hpp"

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
template <typename Call>
auto with_attn_shape(int head_dim, bool f16, AttnForm f, Call call)
{
    if (head_dim == 64) return f16 ? with_attn_shape<64, true>(f, call) : with_attn_shape<64, false>(f, call);
    return f16 ? with_attn_shape<128, true>(f, call) : with_attn_shape<128, false>(f, call);
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
        const void *kernel = (const void *)tree_attn_kernel<S>;
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
hipError_t attn_launch(TreeAttnArgs &a, hipStream_t s)
{
    a.place = (long long *)(a.join + a.groups);
    a.part = (float *)(a.place + (size_t)a.groups * S::TM);
    tree_attn_kernel<S><<<dim3((unsigned)a.groups), dim3(S::THREADS), S::BYTES, s>>>(a);
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
    return with_attn_shape(cache->head_dim, cache->dtype == STAND_F16, f,
                           [&](auto s) { return attn_work_bytes<decltype(s)>(attn_groups_of<decltype(s)>(v)); });
}

extern "C" int stand_tree_attention(stand_handle *h, const stand_cache *cache, int32_t layer, const int32_t *d_len,
                                    const int32_t *d_table, int32_t table_width, const int32_t *d_draft_tok,
                                    const stand_tree_rows *rows, void *d_work, uint64_t work_bytes, void *stream)
{
    if (!h) return STAND_EINVAL;
    const ServeView v = serve_view(h);
    const int refused = check_tree_attention(v.B, cache, layer, d_len, d_table, table_width, d_draft_tok, rows, d_work);
    if (refused) return refused;
    TreeAttnArgs a;
    a.q = (const uint16_t *)rows->d_q; a.k_new = (const uint16_t *)rows->d_k; a.v_new = (const uint16_t *)rows->d_v;
    a.out = (uint16_t *)rows->d_out;
    a.k_pool = (const uint16_t *)cache->d_k + layer * cache->layer_stride;
    a.v_pool = (const uint16_t *)cache->d_v + layer * cache->layer_stride;
    a.len = d_len; a.table = d_table; a.draft_tok = d_draft_tok;
    a.anc = (const uint32_t *)v.anc; a.anc_words = 2 * v.anc_words;      // (little endian: words of 32 nodes)
    a.join = (JoinRecord *)d_work;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = rows->q_stride[i]; a.ks[i] = rows->k_stride[i]; a.vs[i] = rows->v_stride[i]; a.os[i] = rows->out_stride[i];
    }
    a.pool_page = cache->page_stride; a.pool_slot = cache->slot_stride; a.pool_head = cache->head_stride;
    a.scale = rows->scale; a.B = v.B; a.N = v.N; a.kv_heads = cache->kv_heads; a.per_kv = rows->q_heads / cache->kv_heads;
    a.width = table_width; a.pages = cache->pages; a.page_shift = log2_of(cache->page_size);
    return with_attn_shape(cache->head_dim, cache->dtype == STAND_F16, attn_form((int64_t)v.N * a.per_kv), [&](auto s) {
        using S = decltype(s);
        a.groups = attn_groups_of<S>(v);
        if (a.groups == 0) return STAND_EHIP;
        if (work_bytes < attn_work_bytes<S>(a.groups)) return STAND_EINVAL;
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
