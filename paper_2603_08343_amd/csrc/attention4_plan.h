// Argument checks of the cache in 4 bits (include/wht_attention4.h) and of rotary positions of several axes (include/wht_rotary.h).
// Calls are cut as attention_plan.h says.  Compiles without HIP.
#pragma once
#include "../../include/wht_attention4.h"
#include "attention_plan.h"

namespace wht {

// The few-rows kernel takes a sequence's rows of a key head as one or two tiles of 16; pages of 8 tokens have kernels for two alone.
constexpr int kSmallTile = 16;
constexpr int tiles4(int page_size, int own_cap) { return page_size < kSmallTile || own_cap > kSmallTile ? 2 : 1; }

// The few-rows kernel's workgroups, of four workers: three on a compute unit where a worker's registers allow it, else two.  Heads of 128 need more of
// them for the rows they sum up, and have more to do between two loads.  Two / three, in us: 48 sequences of 2 to 5 new tokens and up to 6000 of their own at
// 16 x 96 77 / 71, at 12 x 64 52 / 44; single new tokens, 128 sequences of up to 4096 at 12 x 64 71 / 60, 256 of up to 2048 at 16 and 4 x 64 36 / 32, 64 of up to 8192
// 32 / 27, 200 of up to 2048 at 16 x 96 110 / 103; but one of 65001 at 16 and 4 x 64 15.1 / 16.4, at 12 and 4 x 96 18.7 / 20.6, where the join has half as many pieces again;
// 256 of up to 8192 at 32 and 8 x 128 204 / 212, one of 65001 22.3 / 25.7.
constexpr int workgroups4(bool f32, int head_dim, int tiles, bool front) { return f32 || head_dim == 128 || tiles == 2 || front ? 512 : 768; }
constexpr int kMostWorkers4 = 4 * 768;

// Whether the few-rows kernel reads a call's own codes past the caches: as streams() in attention_plan.h, with a row's bytes here.  Three caches read in turn, kept / past,
// in us: 1 sequence at 32 and 8 x 128, 80 MB 24.3 / 25.1, 96 MB 27.4 / 27.5, 112 MB 31.8 / 30.1, 256 MB 55.9 / 49.8; 16 of them 22.6 / 23.3, 26.9 / 27.0, 31.6 / 29.3,
// 56.5 / 49.9; 128 at 12 x 64 24.7 / 27.7, 33.2 / 33.1, 36.0 / 33.9, 68.3 / 63.5; 16 at 16 and 4 x 64 25.4 / 28.0, 29.6 / 30.6, 36.2 / 34.2, 65.6 / 61.5.
inline bool streams4(int32_t B, int32_t heads, int32_t head_dim, int64_t max_length, int64_t prefix, int32_t gang_log2) {
    return gang_log2 == 0 && ((double)B * max_length + prefix) * heads * (head_dim / 2 + head_dim / 32) * 2 >= 96e6;
}

// Whether a sequence's rows of a key head are taken whole, by a workgroup, in one launch: where all of these have a place at the same time, and the longest that
// lengths can be is short, the shorter the fewer they are.  On the line with its join / whole, in us, sequences of 3/4 of that length and more, 32 and 8 x 128: 8 items
// of up to 128 keys 9.7 / 6.9, 512 10.4 / 8.4, 1024 10.4 / 10.7; 32 of 512 10.9 / 8.8, 1024 11.1 / 11.1, 2048 13.0 / 15.5; 128 of 1024 14.1 / 11.5, 2048 17.0 / 16.2,
// 4096 21.2 / 24.3; 256 of 512 15.2 / 9.3, 2048 22.4 / 17.5, 4096 32.3 / 26.7.  512 items have two rounds (512 keys 19.5 / 18.0), but of 64 wide, two to a
// compute unit (512 keys 17.1 / 9.5, 2048 24.7 / 18.4).  The line deals ragged lengths out evenly, which a workgroup an item does not: lengths from 1 to the
// longest take it the time of half of that, so that the rule stops where those break even.
inline bool takes_whole(int64_t items, int32_t head_dim, int64_t keys) {
    return items > 0 && items <= (head_dim == 64 ? 512 : 256) && keys <= 512 + 8 * (items < 256 ? items : 256);
}
struct AttentionPlan4 : AttentionPlan { bool whole; };
inline AttentionPlan4 plan_attention4(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q, int64_t max_length, int64_t prefix) {
    AttentionPlan4 p{plan_attention(T, B, q_heads, heads, head_dim, max_q, max_length, prefix, kMostWorkers4), false};
    p.whole = p.own_few && !p.front && takes_whole((int64_t)B * heads, head_dim, max_length + prefix);
    if (p.whole) { p.combine = false; p.bytes = 0; }
    return p;
}

constexpr int kMaxPairs = WHT_ROTARY_MAX_HEAD / 2;

// rotary > 0: whether every pair's axis is one of those that positions have.
inline bool good_axes(const uint8_t* pair_axes, int rotary, int axes) {
    for (int i = 0; pair_axes && i < rotary / 2; ++i)
        if (pair_axes[i] >= axes) return false;
    return true;
}

inline int check_rotary(const wht_attention_rows_t* x, const wht_attention_rows_t* out, int64_t T, int32_t heads, int32_t head_dim, const float* rope,
                        int64_t rope_rows, int32_t rotary, const int32_t* positions, int32_t axes, const uint8_t* pair_axes, int32_t dtype) {
    if (!x || !out || !x->data || !out->data || !rope) return WHT_ERR_NULL_PTR;
    if (dtype != WHT_DTYPE_F32 && dtype != WHT_DTYPE_BF16) return WHT_ERR_BAD_DTYPE;
    if (T < 0 || T > (int64_t)1 << 30 || heads < 1 || heads > 1024 || head_dim < 16 || head_dim > WHT_ROTARY_MAX_HEAD || head_dim % 16 != 0) return WHT_ERR_BAD_DIM;
    if (rotary < 16 || rotary % 16 != 0 || rotary > head_dim || rope_rows < 0 || rope_rows > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    if (axes < 1 || axes > WHT_ROTARY_MAX_AXES || (!positions && axes != 1) || !good_axes(pair_axes, rotary, axes)) return WHT_ERR_BAD_DIM;
    const int size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    if (!good_rows(x, heads, head_dim, size) || !good_rows(out, heads, head_dim, size) || ((uintptr_t)rope & 15u) != 0 || ((uintptr_t)positions & 3u) != 0) return WHT_ERR_MISALIGNED;
    if (!apart({T, out->token_stride}, {heads, out->head_stride}, {1, 0}, head_dim)) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

inline int check_cache4(const wht_attention_cache4_t* c, const wht_attention_batch_t* b, int32_t dtype) {
    if (!c || !b || !c->k || !c->v || !c->k_scales || !c->v_scales || !b->table || !b->lengths) return WHT_ERR_NULL_PTR;
    if (dtype != WHT_DTYPE_F32 && dtype != WHT_DTYPE_BF16) return WHT_ERR_BAD_DTYPE;
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return WHT_ERR_BAD_DIM;
    if (c->page_size < WHT_ATTENTION_MIN_PAGE || c->page_size > WHT_ATTENTION_MAX_PAGE || (c->page_size & (c->page_size - 1)) != 0) return WHT_ERR_BAD_DIM;
    if (c->heads < 1 || c->heads > 1024 || c->pages < 1 || b->B < 0 || b->B > 1 << 30 || b->width < 1 || b->table_stride < 0) return WHT_ERR_BAD_DIM;
    if ((int64_t)b->width * c->page_size > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    // a page's number is multiplied by its stride in bytes (both 32 bits), and a row's place in its page stays below 31
    auto fits = [&](int64_t page, int64_t head, int64_t token, int row) {
        return page >= 0 && page < (int64_t)1 << 32 && token >= row && token < (int64_t)1 << 31 && (c->page_size - 1) * token < (int64_t)1 << 31 && head >= 0;
    };
    if (!fits(c->page_stride, c->head_stride, c->token_stride, c->head_dim / 2) ||
        !fits(c->scale_page_stride, c->scale_head_stride, c->scale_token_stride, c->head_dim / 32)) return WHT_ERR_BAD_DIM;
    if (((uintptr_t)c->k & 15u) != 0 || ((uintptr_t)c->v & 15u) != 0 || c->page_stride % 16 != 0 || c->head_stride % 16 != 0 || c->token_stride % 16 != 0) return WHT_ERR_MISALIGNED;
    if (((uintptr_t)b->table & 3u) != 0 || ((uintptr_t)b->lengths & 3u) != 0 || ((uintptr_t)b->q_starts & 3u) != 0) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

inline int check_append4(const wht_attention_rows_t* q, const wht_attention_rows_t* k, const wht_attention_rows_t* v, const wht_attention_rows_t* q_out,
                         const wht_attention_rows_t* k_out, const wht_attention_rows_t* v_out, int64_t T, int32_t q_heads, const wht_attention_cache4_t* c,
                         const wht_attention_batch_t* b, const float* rope, int64_t rope_rows, int32_t rotary, int64_t position, const int32_t* positions,
                         int32_t axes, const uint8_t* pair_axes, int32_t dtype) {
    if (!q || !k || !v || !q_out || !k_out || !v_out || !k->data || !v->data || (q->data && !q_out->data) || (rotary != 0 && !rope)) return WHT_ERR_NULL_PTR;
    if (!k_out->data != !v_out->data) return WHT_ERR_NULL_PTR;
    if (int rc = check_cache4(c, b, dtype)) return rc;
    const int size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    if (T < 0 || T > (int64_t)1 << 30 || (q->data && (q_heads < 1 || q_heads > 1024))) return WHT_ERR_BAD_DIM;
    if (rotary < 0 || rotary % 16 != 0 || rotary > c->head_dim || rope_rows < 0 || rope_rows > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    if (position < 0 || position > (int64_t)1 << 30) return WHT_ERR_BAD_DIM;
    if (axes < 1 || axes > WHT_ROTARY_MAX_AXES || (!positions && axes != 1) || !good_axes(pair_axes, rotary, axes)) return WHT_ERR_BAD_DIM;
    if (!good_rows(k, c->heads, c->head_dim, size) || !good_rows(v, c->heads, c->head_dim, size) || ((uintptr_t)rope & 15u) != 0 || ((uintptr_t)positions & 3u) != 0) return WHT_ERR_MISALIGNED;
    if (q->data && (!good_rows(q, q_heads, c->head_dim, size) || !good_rows(q_out, q_heads, c->head_dim, size))) return WHT_ERR_MISALIGNED;
    if (q->data && !apart({T, q_out->token_stride}, {q_heads, q_out->head_stride}, {1, 0}, c->head_dim)) return WHT_ERR_MISALIGNED;
    if (k_out->data)
        for (const wht_attention_rows_t* r : {k_out, v_out})
            if (!good_rows(r, c->heads, c->head_dim, size) || !apart({T, r->token_stride}, {c->heads, r->head_stride}, {1, 0}, c->head_dim)) return WHT_ERR_MISALIGNED;
    if (!apart({c->pages, c->page_stride}, {c->heads, c->head_stride}, {c->page_size, c->token_stride}, c->head_dim / 2) ||
        !apart({c->pages, c->scale_page_stride}, {c->heads, c->scale_head_stride}, {c->page_size, c->scale_token_stride}, c->head_dim / 32)) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

inline int check_paged4(const wht_attention_rows_t* q, const wht_attention_rows_t* out, const float* lse, int64_t T, int32_t q_heads,
                        const wht_attention_cache4_t* c, const wht_attention_batch_t* b, const int32_t* prefix_table, int64_t prefix,
                        int32_t max_q, int64_t max_length, float scale, int32_t dtype) {
    if (!q || !out || !q->data || !out->data || (prefix > 0 && !prefix_table)) return WHT_ERR_NULL_PTR;
    if (int rc = check_cache4(c, b, dtype)) return rc;
    if (int rc = check_sizes(T, b->B, q_heads, c->heads, c->head_dim, max_q, max_length, prefix, dtype)) return rc;
    if (!(scale > 0.0f) || !(base2_scale(scale) < __builtin_inff())) return WHT_ERR_BAD_DIM;
    // the few-rows kernel counts the blocks of its line in 31 bits
    const int64_t own = (int64_t)b->width * c->page_size < max_length ? (int64_t)b->width * c->page_size : max_length;
    if (((int64_t)b->B + 1) * (own / kBlockKeys + prefix / kBlockKeys + 2) > INT32_MAX / c->heads) return WHT_ERR_BAD_DIM;
    const int size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    if (!good_rows(q, q_heads, c->head_dim, size) || !good_rows(out, q_heads, c->head_dim, size)) return WHT_ERR_MISALIGNED;
    if (!apart({T, out->token_stride}, {q_heads, out->head_stride}, {1, 0}, c->head_dim)) return WHT_ERR_MISALIGNED;
    if (((uintptr_t)lse & 3u) != 0 || ((uintptr_t)prefix_table & 3u) != 0) return WHT_ERR_MISALIGNED;
    return WHT_OK;
}

}  // namespace wht
