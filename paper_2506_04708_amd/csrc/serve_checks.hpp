// serve_checks.hpp -- what the operators around a verification accept (include/stand.h), in plain host code: each check gives
// the code that its call returns before anything is launched.
#pragma once
#include "../../include/stand.h"
#include "attn_plan.hpp"

#include <cmath>
#include <cstring>

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

inline bool of_four(const stand_cache *c) { return c->dtype == STAND_MXFP4 + STAND_BF16 || c->dtype == STAND_MXFP4 + STAND_F16; }
inline int rows_dtype(const stand_cache *c) { return of_four(c) ? c->dtype - STAND_MXFP4 : c->dtype; }
inline const stand_cache4 *four_of(const stand_cache *c) { return reinterpret_cast<const stand_cache4 *>(c); }   // (its first member)
// Scales of a cache of 4 bits: a head's stand together.
inline bool scales_ok(const stand_cache *c)
{
    const stand_cache4 *f = four_of(c);
    const int64_t unit = c->head_dim / 32;
    auto ok = [&](int64_t s) { return s >= 0 && s % unit == 0 && s < ((int64_t)1 << 48); };
    return f->d_k_scale && f->d_v_scale && (uintptr_t)f->d_k_scale % unit == 0 && (uintptr_t)f->d_v_scale % unit == 0 && ok(f->scale_layer_stride) &&
           ok(f->scale_page_stride) && ok(f->scale_slot_stride) && ok(f->scale_head_stride) && c->layer_stride % 32 == 0 &&
           c->page_stride % 32 == 0 && c->slot_stride % 32 == 0 && c->head_stride % 32 == 0;
}

inline bool cache_ok(const stand_cache *c)
{
    return c && c->d_k && c->d_v && aligned16(c->d_k) && aligned16(c->d_v) && (c->dtype == STAND_BF16 || c->dtype == STAND_F16 || of_four(c)) &&
           c->layers >= 1 && c->pages >= 1 && page_size_ok(c->page_size) && c->kv_heads >= 1 && c->kv_heads <= 4096 &&
           (c->head_dim == 64 || c->head_dim == 128) && stride_ok(c->layer_stride) && stride_ok(c->page_stride) &&
           stride_ok(c->slot_stride) && stride_ok(c->head_stride) && (!of_four(c) || scales_ok(c));
}

// Whether places (x, y) up to these lie less than 2^32 chunks of that many elements from the first one (x, y < 2^31).
inline bool spans_chunks(int64_t x, int64_t x_stride, int64_t y, int64_t y_stride, int64_t chunk = 8)
{
    const int64_t most = (int64_t)1 << 32, xs = x_stride / chunk, ys = y_stride / chunk;
    if ((x && xs >= most / x) || (y && ys >= most / y)) return false;
    return x * xs + y * ys < most - 64;
}

inline bool heads_ok(const stand_cache *c, int32_t q_heads) { return q_heads >= 1 && q_heads % c->kv_heads == 0; }

// Whether there is an attention of that size at all: what its workspace depends on, and how far it can count.
inline int check_attention_size(int64_t B, const stand_cache *cache, int32_t q_heads)
{
    if (!cache_ok(cache) || !heads_ok(cache, q_heads)) return STAND_EINVAL;
    if (B > kAttnMaxBatch || q_heads > 65535) return STAND_ELIMIT;
    // the kernel counts places of a layer in 16-byte chunks, in 32 bits, and those of scales in heads' scales
    if (!spans_chunks(cache->pages - 1, cache->page_stride, cache->page_size - 1, cache->slot_stride, of_four(cache) ? 32 : 8)) return STAND_ELIMIT;
    if (of_four(cache) && !spans_chunks(cache->pages - 1, four_of(cache)->scale_page_stride, cache->page_size - 1, four_of(cache)->scale_slot_stride,
                                         cache->head_dim / 32))
        return STAND_ELIMIT;
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

// Places that are written differ from each other (a view that repeats one, as torch's expand makes them, would be written by many).
inline bool apart(int64_t stride, int64_t count) { return stride != 0 || count == 1; }

inline int check_cache_read(int64_t B, const stand_cache *cache, int32_t first_layer, int32_t layers, const int32_t *d_table, int32_t table_width,
                            const stand_cache_rows_out *rows)
{
    if (!cache_ok(cache) || !rows || !rows->d_k || !rows->d_v || !d_table || table_width < 1) return STAND_EINVAL;
    if (first_layer < 0 || layers < 1 || layers > cache->layers || first_layer > cache->layers - layers) return STAND_EINVAL;
    if (rows->rows < 1 || rows->rows > kServeMaxWidth || (int64_t)table_width * cache->page_size > STAND_MAX_CACHED) return STAND_EINVAL;
    if (!aligned16(rows->d_k) || !aligned16(rows->d_v)) return STAND_EINVAL;
    if (!stride_ok(rows->layer_stride) || !stride_ok(rows->batch_stride) || !stride_ok(rows->row_stride) || !stride_ok(rows->head_stride))
        return STAND_EINVAL;
    if (!apart(rows->layer_stride, layers) || !apart(rows->batch_stride, B) || !apart(rows->row_stride, rows->rows) ||
        !apart(rows->head_stride, cache->kv_heads))
        return STAND_EINVAL;
    return B > kServeMaxBatch || layers > 65535 ? STAND_ELIMIT : STAND_OK;
}

inline bool rotation_ok(const stand_rotation *r, int32_t head_dim)
{
    if (!r || r->dims < 0 || r->dims % 16 || r->dims > head_dim || (r->dims && (!r->d_turns || !aligned16(r->d_turns) || r->positions < 1))) return false;
    if (!aligned16(r->d_q_norm) || !aligned16(r->d_k_norm)) return false;
    return !(r->d_q_norm || r->d_k_norm) || (r->eps >= 0.0f && r->eps <= 3.402823466e+38f);
}

// An output [B][rows][heads] is its input in the same places, or somewhere else.
inline bool output_ok(const void *out, const int64_t *out_stride, const void *in, const int64_t *in_stride, int64_t B, int64_t rows, int64_t heads)
{
    return out && aligned16(out) && strides_ok(out_stride) && apart(out_stride[0], B) && apart(out_stride[1], rows) && apart(out_stride[2], heads) &&
           (out != in || !memcmp(out_stride, in_stride, 3 * sizeof(int64_t)));
}

constexpr int64_t kTurnMaxGroups = (1 << 24) - 1;      // workgroups of a trajectory: a launch's dimension has threads for so many
inline int64_t turn_groups(int64_t rows, int64_t heads, int32_t head_dim)
{
    const int64_t at_once = 256 / (head_dim / 16);
    return (rows * heads + at_once - 1) / at_once;
}

inline int check_turned_rows(int64_t B, const stand_turned_rows *r, bool values, bool k_out)
{
    if (!r || !r->d_k || !aligned16(r->d_k) || !strides_ok(r->k_stride)) return STAND_EINVAL;
    if ((r->dtype != STAND_BF16 && r->dtype != STAND_F16) || (r->head_dim != 64 && r->head_dim != 128)) return STAND_EINVAL;
    if (r->rows < 1 || r->rows > kServeMaxWidth || r->kv_heads < 1 || r->kv_heads > 4096) return STAND_EINVAL;
    if (r->d_q && (r->q_heads < 1 || !aligned16(r->d_q) || !strides_ok(r->q_stride) || !output_ok(r->d_q_out, r->q_out_stride, r->d_q, r->q_stride, B, r->rows, r->q_heads)))
        return STAND_EINVAL;
    if ((k_out || r->d_k_out) && !output_ok(r->d_k_out, r->k_out_stride, r->d_k, r->k_stride, B, r->rows, r->kv_heads)) return STAND_EINVAL;
    if (values && (!r->d_v || !aligned16(r->d_v) || !strides_ok(r->v_stride))) return STAND_EINVAL;
    if (B > kServeMaxBatch || (r->d_q && r->q_heads > 65535)) return STAND_ELIMIT;
    const int64_t q = r->d_q ? turn_groups(r->rows, r->q_heads, r->head_dim) : 0, k = turn_groups(r->rows, r->kv_heads, r->head_dim);
    return q + k + (values ? k : 0) > kTurnMaxGroups ? STAND_ELIMIT : STAND_OK;
}

inline int check_tree_rotate(int64_t B, int32_t N, const stand_rotation *rotation, const int32_t *d_len, const int32_t *d_draft_tok,
                             const stand_turned_rows *rows)
{
    if (!rows || (rows->head_dim != 64 && rows->head_dim != 128) || !rotation_ok(rotation, rows->head_dim) || !d_len || !d_draft_tok) return STAND_EINVAL;
    if (rows->rows != N) return STAND_EINVAL;
    return check_turned_rows(B, rows, false, true);
}

inline int check_cache_append(int64_t B, const stand_cache *cache, int32_t layer, const stand_rotation *rotation, const stand_turned_rows *rows,
                              const int64_t *d_slots, int32_t width)
{
    if (!cache_ok(cache) || !rows || layer < 0 || layer >= cache->layers || !d_slots) return STAND_EINVAL;
    if (rows->dtype != rows_dtype(cache) || rows->kv_heads != cache->kv_heads || rows->head_dim != cache->head_dim) return STAND_EINVAL;
    if ((rotation && !rotation_ok(rotation, rows->head_dim)) || width < rows->rows || width > kServeMaxWidth) return STAND_EINVAL;
    return check_turned_rows(B, rows, true, false);
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
