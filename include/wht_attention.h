/*
 * wht_attention.h -- C ABI of the paged cache and the attention in front of the Walsh-Hadamard output layer
 * (wht_affine.h) for AMD MI355X (gfx950): what supplies the concatenated head outputs x[N,:] that the layer transforms.
 *
 * The cache.  Keys and values of all sequences lie in pages of `page_size` tokens:
 *
 *     k[page][head][slot][0 .. head_dim)        at  k + page * page_stride + head * head_stride + slot * token_stride   (elements)
 *
 * and v likewise with the same strides, so that [pages][heads][page_size][head_dim] and [pages][page_size][heads][head_dim] are both
 * taken as they are.  A sequence's tokens stand in the pages that its row of `table` names, in order: its token p in
 * page table[b][p / page_size], slot p % page_size.
 *
 * The batch.  B sequences; lengths[b] counts the tokens of sequence b that are its own, the new ones included and last.
 * The new tokens' rows are packed: those of sequence b are rows q_starts[b] .. q_starts[b+1)-1 of q, k, v and of the
 * outputs; without q_starts every sequence has one new token, row b.  Rows from q_starts[B] on belong to no sequence (padding).
 *
 * Append.  New token j of the n_b new ones of sequence b is its own token p = lengths[b] - n_b + j and has the position
 * position + p.  With the angles' cosine c and sine s of that position (rope[position][i] = {c, s}, i < rotary / 2):
 *
 *     (x_a, x_b)  ->  (x_a c - x_b s,  x_b c + x_a s)      a, b = i, i + rotary / 2   (or 2 i, 2 i + 1 where `interleaved`)
 *
 * for every head of q and k, in float32, rounded once (to nearest even); elements from `rotary` on, and v, are copied.
 * k and v go to the token's place in the cache, q to q_out.
 *
 * Attention.  Every token of the batch sees the `prefix_length` tokens in the pages of prefix_table -- one prefix, shared by all
 * sequences -- and of its own sequence the tokens 0 .. p:
 *
 *     s_t = scale * <q, k_t>       out = sum_t exp(s_t) v_t / sum_t exp(s_t)       lse = log sum_t exp(s_t)
 *
 * over the keys t that it sees.  Query head h reads key head h / (q_heads / heads).  Sums, maxima and the scores are float32;
 * for bfloat16 tensors the weights are rounded to bfloat16 for the product with v (their sum is not).  A token that sees
 * nothing has out = 0 and lse = -inf.
 *
 * What lies in a place that no token sees has no influence, whatever it holds (infinities and NaN as well).  The kernels
 * look at the device arrays' values before they use them:
 *   - a page number outside [0, pages) names no memory: nothing is stored there, and its tokens count as not there;
 *   - attention takes lengths within [0, width * page_size] and up to max_length;
 *   - a token without a place in the cache (no sequence, p < 0, p past the table) is not stored;
 *   - a position outside the rows of `rope` is not stored either, and its row of q_out is NaN;
 *   - a row of q that belongs to no sequence gives a row of zeros (append and attention; lse = -inf);
 *   - a token from the max_q-th of its sequence on, where max_q is too small, gives a row of NaN.
 *
 * Conventions for both entry points: device pointers; `stream` is a hipStream_t (NULL: the default stream); nothing is allocated or
 * synchronised; the arguments are validated before anything is enqueued; both may be captured into a HIP graph, which then replays
 * with the arrays' new values.  Results are bit-reproducible.  Outputs may not overlap inputs, except that the append's
 * q_out may be q itself; nor themselves (strides that let them are refused, those of a cache that is appended to as well).
 */
#ifndef WHT_ATTENTION_H
#define WHT_ATTENTION_H

#include <stddef.h>
#include <stdint.h>

#include "wht_affine.h"      /* wht_dtype_t, wht_status_t */

#ifdef __cplusplus
extern "C" {
#endif

#define WHT_ATTENTION_MIN_PAGE 8
#define WHT_ATTENTION_MAX_PAGE 1024

/* A tensor [rows][heads][head_dim], the last dimension contiguous; strides in elements. */
typedef struct {
    void *data;
    int64_t token_stride, head_stride;
} wht_attention_rows_t;

typedef struct {
    void *k, *v;                                        /* 16-byte aligned */
    int64_t page_stride, head_stride, token_stride;     /* in elements, of k and of v; 16-byte steps */
    int32_t pages, heads, page_size, head_dim;          /* page_size: a power of two, 8 .. 1024; head_dim: 64, 96, 128 */
} wht_attention_cache_t;

typedef struct {
    const int32_t *table;           /* [B][width], rows table_stride apart */
    const int32_t *lengths;         /* [B] */
    const int32_t *q_starts;        /* [B + 1], ascending from 0; NULL: one new token each */
    int64_t table_stride;
    int32_t B, width;
} wht_attention_batch_t;

/*
 * Append the new tokens of a batch to the cache (see the header comment).
 *   q        in    T rows of q_heads heads, or data = NULL: no queries (q_out is then not used)
 *   k, v     in    T rows of cache->heads heads
 *   q_out    out   T rows of q_heads heads
 *   rope     in    [rope_rows][rotary / 2][2] float32, contiguous; NULL (rotary = 0): no rotation
 *   rotary         0, or a multiple of 16 up to head_dim
 *   position       of a sequence's first own token: the length of the prefix before it
 */
int wht_attention_append(const wht_attention_rows_t *q, const wht_attention_rows_t *k, const wht_attention_rows_t *v,
                         const wht_attention_rows_t *q_out, int64_t T, int32_t q_heads,
                         const wht_attention_cache_t *cache, const wht_attention_batch_t *batch,
                         const float *rope, int64_t rope_rows, int32_t rotary, int32_t interleaved, int64_t position,
                         int32_t dtype, void *stream);

/*
 * Bytes of device scratch that wht_attention_paged needs for such a call: partial results of rows whose keys several workgroups
 * share.  Depends on these arguments alone; 0 for T = 0 or invalid ones.  Needs no GPU.
 */
size_t wht_attention_workspace_bytes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim,
                                     int32_t max_q, int64_t max_length, int64_t prefix_length, int32_t dtype);

/*
 * Attention of the new tokens over the prefix and their own sequences (see the header comment).
 *   q             in    T rows of q_heads heads, q_heads a multiple of cache->heads
 *   out           out   T rows of q_heads heads
 *   lse           out   [T][q_heads] float32, or NULL
 *   prefix_table  in    [ceil(prefix_length / page_size)], NULL where prefix_length = 0
 *   max_q               at least the largest number of new tokens of a sequence
 *   max_length          at least the largest of lengths; how the work is split goes by it (width * page_size always does)
 *   scale               > 0, at most 2.3e38 (its product with log2(e) is finite)
 *   workspace           device scratch, 16-byte aligned, at least ..._workspace_bytes(...) bytes; contents on entry are ignored
 */
int wht_attention_paged(const wht_attention_rows_t *q, const wht_attention_rows_t *out, float *lse, int64_t T, int32_t q_heads,
                        const wht_attention_cache_t *cache, const wht_attention_batch_t *batch,
                        const int32_t *prefix_table, int64_t prefix_length, int32_t max_q, int64_t max_length, float scale,
                        int32_t dtype, void *workspace, size_t workspace_bytes, void *stream);

/* Static, NUL-terminated description of a status of these entry points. */
const char *wht_attention_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* WHT_ATTENTION_H */
