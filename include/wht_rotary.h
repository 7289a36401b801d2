/*
 * wht_rotary.h -- C ABI of rotary positions of several axes (time, height and width of pictures and video) for AMD MI355X
 * (gfx950), in front of attention: in training, and of queries and keys that go into a cache.
 *
 * A token t has a position on each of `axes` axes, positions[t][0 .. axes).  The pair i < rotary / 2 of every head turns by the angle of
 * the position on its own axis pair_axes[i], whose cosine c and sine s stand in rope[position][i] = {c, s}:
 *
 *     (x_a, x_b)  ->  (x_a c - x_b s,  x_b c + x_a s)      a, b = i, i + rotary / 2   (or 2 i, 2 i + 1 where `interleaved`)
 *
 * in float32, rounded once (to nearest even); elements from `rotary` on are copied.  `inverse` turns back (s -> -s), which is also the
 * gradient: of y = R x it is dx = R^T dy.
 *
 * A position outside the rows of `rope` on the axis of any pair gives a row of NaN, in every head.
 *
 * Conventions as in wht_attention.h: device pointers (pair_axes aside); nothing is allocated or synchronised; arguments are validated before
 * anything is enqueued; the call may be captured into a HIP graph (pair_axes is read during the call, and part of what is captured).
 */
#ifndef WHT_ROTARY_H
#define WHT_ROTARY_H

#include "wht_attention.h"      /* wht_attention_rows_t */

#ifdef __cplusplus
extern "C" {
#endif

#define WHT_ROTARY_MAX_AXES 4
#define WHT_ROTARY_MAX_HEAD 256

/*
 *   x           in    T rows of `heads` heads of head_dim elements (a multiple of 16, up to WHT_ROTARY_MAX_HEAD)
 *   out         out   the same; x itself, with its strides, or no overlap with it
 *   rope        in    [rope_rows][rotary / 2][2] float32, contiguous; rotary a multiple of 16 up to head_dim, at least 16
 *   positions   in    [T][axes] int32, contiguous; NULL (axes = 1): token t has position t
 *   pair_axes   in    HOST memory, [rotary / 2] numbers below `axes`; NULL: all 0
 */
int wht_rotary_rotate(const wht_attention_rows_t *x, const wht_attention_rows_t *out, int64_t T, int32_t heads, int32_t head_dim,
                      const float *rope, int64_t rope_rows, int32_t rotary, int32_t interleaved,
                      const int32_t *positions, int32_t axes, const uint8_t *pair_axes, int32_t inverse, int32_t dtype, void *stream);

/* Static, NUL-terminated description of a status of this entry point. */
const char *wht_rotary_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* WHT_ROTARY_H */
