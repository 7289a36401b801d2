/*
 * wht_attention4.h -- C ABI of the paged cache in 4 bits and its attention for AMD MI355X (gfx950): what wht_attention.h
 * does with a cache of 16- or 32-bit numbers, with keys and values of half a byte and a scale byte for every 32 of them.
 *
 * The numbers.  A code of 4 bits is a sign (bit 3) and a magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0 .. 2).  Element 2 i of a row stands in
 * the low half of its byte i, 2 i + 1 in the high half.  A block is 32 elements of a head, from a multiple of 32 on; its scale byte e stands
 * for 2^(e - 127), and from 253 on for "not a number": all 32 are NaN then.
 *
 * The cache.  Pages as in wht_attention.h, once for codes, once for scales:
 *
 *     k[page][head][slot][0 .. head_dim / 2)           at  k + page * page_stride + head * head_stride + slot * token_stride     (bytes)
 *     k_scales[page][head][slot][0 .. head_dim / 32)   at  k_scales + page * scale_page_stride + ...                             (bytes)
 *
 * and v, v_scales likewise with the same strides.  Tables, lengths, batch and rows are those of wht_attention.h.
 *
 * Append.  A new token's queries and keys are rotated: by its position in its sequence as wht_attention_append does it, or, with `positions`,
 * by those on several axes as wht_rotary_rotate does it.  Then, where `transform`, every block passes a Walsh-Hadamard transform with entries
 * +-1 (Sylvester order, H of 32), which spreads a large element over the 32 that share a scale:
 *
 *     q' = H q / 8      k' = H k / 4      v' = H v / 4         so that <q', k'> = <q, k>  and  H v' / 8 = v
 *
 * q' is computed in float32 and rounded once; k' and v' are computed in 64 bits, and stored as the codes nearest to them (of two as near the
 * even one; a zero has no sign), with the least scale 2^e, -124 <= e <= 125, for which 6 * 2^e is no less than any magnitude of the block (a larger
 * magnitude than 6 * 2^125 becomes that).  A block with an element that is not finite is stored as not a number, codes 0.
 *
 * Attention.  As wht_attention_paged, with the numbers that the cache stands for; where `transform`, q is q' as the append gives it and
 * out = H (sum_t p_t v'_t) / 8, in float32, rounded once.  Results have the type of q.  For bfloat16 queries the weights are rounded to bfloat16 for the product with
 * v' (their sum is not); float32 queries and their weights enter the products with 24 bits (what is below 2^-109 of them as a multiple of 2^-133).  The sums in front of
 * the division by the sum of the weights are float32: of values with scales up to 2^80 (byte 207) they are finite for any number of keys, of larger ones they may not be.
 *
 * What is said there of page numbers, lengths, places, positions and padding rows holds here too; the value of a token that a
 * row does not see takes no part in that row, whatever its bytes.  So do the conventions of its entry points.
 */
#ifndef WHT_ATTENTION4_H
#define WHT_ATTENTION4_H

#include "wht_attention.h"
#include "wht_rotary.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    void *k, *v;                                        /* 16-byte aligned */
    uint8_t *k_scales, *v_scales;
    int64_t page_stride, head_stride, token_stride;     /* bytes, of k and of v; 16-byte steps */
    int64_t scale_page_stride, scale_head_stride, scale_token_stride;       /* bytes, of k_scales and of v_scales */
    int32_t pages, heads, page_size, head_dim;          /* page_size: a power of two, 8 .. 1024; head_dim: 64, 96, 128 */
} wht_attention_cache4_t;

/*
 * Append the new tokens of a batch to the cache (see the header comment).
 *   q, k, v     in    T rows of q_heads, cache->heads, cache->heads heads; q->data = NULL: no queries (q_out is then not used)
 *   q_out       out   T rows of q_heads heads; may be q
 *   k_out, v_out      out   data = NULL, or T rows of cache->heads heads: the numbers that the stored codes stand for, rounded to `dtype`.  Rows of
 *                     tokens that are not stored are NaN, of padding zero.  Not k or v.
 *   rope        in    [rope_rows][rotary / 2][2] float32, contiguous; NULL (rotary = 0): no rotation
 *   rotary            0, or a multiple of 16 up to head_dim
 *   position          of a sequence's first own token; not used with `positions`
 *   positions   in    [T][axes] int32, contiguous, or NULL: one axis, by the token's place
 *   pair_axes   in    HOST memory, [rotary / 2] numbers below `axes`; NULL: all 0
 */
int wht_attention_append4(const wht_attention_rows_t *q, const wht_attention_rows_t *k, const wht_attention_rows_t *v,
                          const wht_attention_rows_t *q_out, const wht_attention_rows_t *k_out, const wht_attention_rows_t *v_out,
                          int64_t T, int32_t q_heads, const wht_attention_cache4_t *cache, const wht_attention_batch_t *batch,
                          const float *rope, int64_t rope_rows, int32_t rotary, int32_t interleaved, int64_t position,
                          const int32_t *positions, int32_t axes, const uint8_t *pair_axes, int32_t transform, int32_t dtype, void *stream);

/*
 * Bytes of device scratch that wht_attention_paged4 needs for such a call (see wht_attention_workspace_bytes).  More sequences, rows or keys may need fewer: 8 sequences of
 * up to 2560 keys at 8 key heads need megabytes, 32 of them, which are taken whole, none.  A workspace for calls of several sizes has the largest of their needs.
 */
size_t wht_attention4_workspace_bytes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t head_dim,
                                      int32_t max_q, int64_t max_length, int64_t prefix_length, int32_t dtype);

/* Attention of the new tokens over the prefix and their own sequences: arguments as of wht_attention_paged; dtype: of q and out. */
int wht_attention_paged4(const wht_attention_rows_t *q, const wht_attention_rows_t *out, float *lse, int64_t T, int32_t q_heads,
                         const wht_attention_cache4_t *cache, const wht_attention_batch_t *batch,
                         const int32_t *prefix_table, int64_t prefix_length, int32_t max_q, int64_t max_length, float scale,
                         int32_t transform, int32_t dtype, void *workspace, size_t workspace_bytes, void *stream);

/* Static, NUL-terminated description of a status of these entry points. */
const char *wht_attention4_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* WHT_ATTENTION4_H */
