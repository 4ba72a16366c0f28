// serve_checks.hpp -- what the operators around a verification accept (include/stand.h), in plain host code: each check gives
// the code that its call returns before anything is launched.
#pragma once
#include "../../include/stand.h"
#include "attn_plan.hpp"

#include <cmath>

namespace stand {

constexpr int kServeMaxBatch = 65535;                  // trajectories: a grid's second dimension
constexpr int32_t kServeMaxWidth = STAND_MAX_CACHED;   // of tables, slots and lists: threads step over them in 32 bits

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0 && s < ((int64_t)1 << 48); }
inline bool strides_ok(const int64_t *s) { return stride_ok(s[0]) && stride_ok(s[1]) && stride_ok(s[2]); }
inline bool page_size_ok(int32_t p) { return p > 0 && (p & (p - 1)) == 0 && p <= STAND_MAX_PAGE; }
inline int log2_of(int64_t x)
{
    int s = 0;
    while (((int64_t)1 << s) < x) ++s;
    return s;
}

inline bool cache_ok(const stand_cache *c)
{
    return c && c->d_k && c->d_v && aligned16(c->d_k) && aligned16(c->d_v) && (c->dtype == STAND_BF16 || c->dtype == STAND_F16) &&
           c->layers >= 1 && c->pages >= 1 && page_size_ok(c->page_size) && c->kv_heads >= 1 && c->kv_heads <= 4096 &&
           (c->head_dim == 64 || c->head_dim == 128) && stride_ok(c->layer_stride) && stride_ok(c->page_stride) &&
           stride_ok(c->slot_stride) && stride_ok(c->head_stride);
}

// Whether places (x, y) up to these lie less than 2^32 chunks of eight elements from the first one (x, y < 2^31).
inline bool spans_chunks(int64_t x, int64_t x_stride, int64_t y, int64_t y_stride)
{
    const int64_t most = (int64_t)1 << 32, xs = x_stride / 8, ys = y_stride / 8;
    if ((x && xs >= most / x) || (y && ys >= most / y)) return false;
    return x * xs + y * ys < most - 64;
}

inline bool heads_ok(const stand_cache *c, int32_t q_heads) { return q_heads >= 1 && q_heads % c->kv_heads == 0; }

// Whether there is an attention of that size at all: what its workspace depends on, and how far it can count.
inline int check_attention_size(int64_t B, const stand_cache *cache, int32_t q_heads)
{
    if (!cache_ok(cache) || !heads_ok(cache, q_heads)) return STAND_EINVAL;
    if (B > kAttnMaxBatch || q_heads > 65535) return STAND_ELIMIT;
    // the kernel counts places of a layer in 16-byte chunks, in 32 bits
    if (!spans_chunks(cache->pages - 1, cache->page_stride, cache->page_size - 1, cache->slot_stride)) return STAND_ELIMIT;
    return STAND_OK;
}

inline int check_tree_attention(int64_t B, const stand_cache *cache, int32_t layer, const int32_t *d_len, const int32_t *d_table,
                                int32_t table_width, const int32_t *d_draft_tok, const stand_tree_rows *rows, const void *d_work)
{
    if (!cache_ok(cache) || !rows || !d_len || !d_table || !d_draft_tok || !d_work || !aligned16(d_work)) return STAND_EINVAL;
    if (layer < 0 || layer >= cache->layers || table_width < 1) return STAND_EINVAL;
    if (!rows->d_q || !rows->d_k || !rows->d_v || !rows->d_out) return STAND_EINVAL;
    if (!aligned16(rows->d_q) || !aligned16(rows->d_k) || !aligned16(rows->d_v) || !aligned16(rows->d_out)) return STAND_EINVAL;
    if (!strides_ok(rows->q_stride) || !strides_ok(rows->k_stride) || !strides_ok(rows->v_stride) || !strides_ok(rows->out_stride))
        return STAND_EINVAL;
    if (!(rows->scale > 0.0f && rows->scale <= 0x1p127f)) return STAND_EINVAL;   // (its product with log2(e) is a number)
    if ((int64_t)table_width * cache->page_size > STAND_MAX_CACHED) return STAND_EINVAL;
    return check_attention_size(B, cache, rows->q_heads);
}

inline int check_cache_commit(int64_t B, const stand_cache *cache, const stand_cache_rows *rows, const int64_t *d_slots, int32_t width)
{
    if (!cache_ok(cache) || !rows || !rows->d_k || !rows->d_v || !d_slots || width < 1 || width > kServeMaxWidth || rows->rows < 1)
        return STAND_EINVAL;
    if (!aligned16(rows->d_k) || !aligned16(rows->d_v)) return STAND_EINVAL;
    if (!stride_ok(rows->layer_stride) || !stride_ok(rows->batch_stride) || !stride_ok(rows->row_stride) || !stride_ok(rows->head_stride))
        return STAND_EINVAL;
    return B > kServeMaxBatch || cache->layers > 65535 ? STAND_ELIMIT : STAND_OK;
}

inline int check_cache_pages(int64_t B, const stand_pages *p, const int64_t *d_slots, int32_t slot_width, const int32_t *d_missing,
                             const stand_pages *out)
{
    if (!p || !out || !p->d_table || !p->d_ring || !p->d_length || !p->d_held || !p->d_mark || !d_missing) return STAND_EINVAL;
    if (!out->d_length || !out->d_held || !out->d_mark) return STAND_EINVAL;
    if (out->d_table != p->d_table || out->d_ring != p->d_ring || out->width != p->width || out->pages != p->pages || out->page_size != p->page_size)
        return STAND_EINVAL;
    if (p->width < 1 || p->pages < 1 || !page_size_ok(p->page_size)) return STAND_EINVAL;
    if (slot_width < 0 || slot_width > kServeMaxWidth || (slot_width > 0 && !d_slots)) return STAND_EINVAL;
    if ((int64_t)p->width * p->page_size > STAND_MAX_CACHED) return STAND_EINVAL;
    return B > kServeMaxBatch ? STAND_ELIMIT : STAND_OK;
}

inline int check_shape_logits(int64_t B, int logits_dtype, const void *d_logits, const void *d_out, const int32_t *d_draft_tok,
                              const int32_t *d_bias_id, const float *d_bias, int32_t bias_width)
{
    if (!d_logits || !d_out || !d_draft_tok) return STAND_EINVAL;
    if (bias_width < 0 || bias_width > kServeMaxWidth || (bias_width > 0 && (!d_bias_id || !d_bias))) return STAND_EINVAL;
    if (((uintptr_t)d_logits | (uintptr_t)d_out) & (logits_dtype == STAND_F32 ? 3u : 1u)) return STAND_EINVAL;
    return B > kServeMaxBatch ? STAND_ELIMIT : STAND_OK;
}

inline int check_count_tokens(int64_t B, const int32_t *d_count, const int32_t *d_tok, int32_t width)
{
    if (!d_count || !d_tok || width < 1 || width > kServeMaxWidth) return STAND_EINVAL;
    return B > kServeMaxBatch ? STAND_ELIMIT : STAND_OK;
}

}  // namespace stand
