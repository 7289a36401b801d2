// The rules of attention_plan.h and attention4_plan.h for the tests, as a library that the host compiler builds: what a call of a size launches.  Not part of the
// attention's library.
#include "attention4_plan.h"

using namespace wht;

extern "C" {

// most: what lengths are cut to.  out: front, front_few, own_few, front_splits, own_splits, own_cap, waves of a joined row (0: no join, or that of even
// splits), log2 of the heads side by side, keys past the caches.
void wht_query_attention(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q, int64_t max_length, int64_t most,
                         int64_t prefix, int32_t dtype, int64_t head_stride, int64_t* out) {
    const int64_t size = dtype == WHT_DTYPE_F32 ? 4 : 2;
    const AttentionPlan p = plan_attention(T, B, q_heads, heads, head_dim, max_q, max_length, prefix);
    const int gang = p.own_few ? gang_log2_of(heads, head_dim * size, head_stride * size) : 0;
    const int64_t values[] = {p.front, p.front_few, p.own_few, p.front_splits, p.own_splits, p.own_cap, p.own_few ? join_waves(T * q_heads) : 0, gang,
                              p.own_few && streams(B, heads, head_dim, size, most, p.front ? 0 : prefix, gang)};
    for (int64_t v : values) *out++ = v;
}
int32_t wht_query_line_share(int32_t total, int32_t rows, int32_t gang_log2) { return line_share(total, rows, gang_log2); }

// The same of the cache in 4 bits: front, front_few, own_few, whole, front_splits, own_splits, own_cap, join_waves, gang_log2, codes past the caches, tiles of 16 rows,
// workers of the few-rows kernel's line.
void wht_query_attention4(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t max_q, int64_t max_length, int64_t most, int64_t prefix,
                          int32_t dtype, int32_t page_size, int64_t head_stride, int64_t* out) {
    const AttentionPlan4 p = plan_attention4(T, B, q_heads, heads, head_dim, max_q, max_length, prefix);
    const bool line = p.own_few && !p.whole;
    const int gang = line ? gang_log2_of(heads, head_dim / 2, head_stride) : 0, tiles = tiles4(page_size, p.own_cap);
    const bool past = line && dtype != WHT_DTYPE_F32 && page_size >= kSmallTile && streams4(B, heads, head_dim, most, p.front ? 0 : prefix, gang);
    const int64_t values[] = {p.front, p.front_few, p.own_few, p.whole, p.front_splits, p.own_splits, p.own_cap, line ? join_waves(T * q_heads) : 0, gang, past, tiles,
                              4 * workgroups4(dtype == WHT_DTYPE_F32, head_dim, tiles, p.front && !p.front_few)};
    for (int64_t v : values) *out++ = v;
}
int32_t wht_query_line_share4(int32_t total, int32_t rows, int32_t gang_log2, int32_t workers) {
    return workers == kMostWorkers4 ? line_share<kMostWorkers4>(total, rows, gang_log2) : line_share(total, rows, gang_log2);
}

}  // extern "C"
