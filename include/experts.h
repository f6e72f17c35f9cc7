/*
 * experts.h: C ABI of mixtures of feed-forward blocks on MI355X (gfx950): rows
 * (pairs, nodes) go to gated blocks of their own, by species, kind of pair or a
 * router's choice.  The rows are sorted by expert, the experts' blocks run on the
 * sorted rows, and the results come back to their rows with weights.  Each has its
 * gradients.
 *
 * Each of N rows has per_row choices; choice k of row n is slot n * per_row + k.
 * A choice outside 0 .. experts - 1 (-1, say) names no expert: its slot has no
 * sorted row, adds nothing and takes no gradient.  A row may choose an expert
 * more than once; each choice counts.
 *
 * Arrays, types, alignment, overlaps, streams, workspaces, graphs and status codes
 * are as in ffn.h.  N == 0 returns CGTP_OK; what sums over rows is then zero.
 * place, source and offsets are device arrays that ffn_route wrote; entries out of
 * their range read and write nothing out of bounds, but give other results.
 */
#ifndef EXPERTS_H
#define EXPERTS_H

#include <stdint.h>

#include "ffn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most experts, and most choices of a row; N * per_row is at most FFN_MAX_ROWS. */
#define FFN_MAX_EXPERTS 1024

/* ------------------------------------------------------------------ rows sorted by expert and back
 *
 * With S = N * per_row slots, sorted by expert and, within an expert, by slot:
 *   offsets [experts + 1]: sorted rows offsets[e] .. offsets[e + 1] - 1 are expert e's
 *   place [N, per_row]:    the sorted row of each slot, -1 where it names no expert
 *   source [S]:            the slot of each sorted row, -1 from offsets[experts] on
 */

/*
 * Sorts.  index: [N, per_row], contiguous, of 4- or 8-byte signed whole numbers
 * (index_bytes).  CGTP_EINVAL for NULL or misaligned arrays, N < 0, per_row or
 * experts below 1, another index_bytes, overlaps, a workspace that is too small;
 * CGTP_EUNSUP for experts or per_row above FFN_MAX_EXPERTS, S > FFN_MAX_ROWS.
 */
int ffn_route(const void *index, int32_t index_bytes, int64_t N, int32_t per_row, int32_t experts, int32_t *place,
              int32_t *source, int32_t *offsets, void *workspace, int64_t workspace_bytes, void *hip_stream);

/* Workspace bytes of ffn_route; -1 if invalid. */
int64_t ffn_route_workspace_bytes(int64_t N, int32_t per_row, int32_t experts);

/*
 * xs [S, width] = the rows of x [N, width] (row stride ldx) in the sorted order:
 * row p is row source[p] / per_row of x; zeros from offsets[experts] on.
 */
int ffn_route_gather(const void *x, int64_t ldx, const int32_t *place, const int32_t *offsets, void *xs, int64_t N,
                     int32_t per_row, int32_t experts, int64_t width, int32_t dtype, void *hip_stream);

/*
 * y [N, width] (row stride ldy): y[n] = sum over k of weights[n, k] * ys[place[n, k]],
 * ys [S, width] in the sorted order; slots without an expert add nothing, whatever
 * their weight.  weights: [N, per_row] 32-bit floats; NULL: ones, which makes this
 * the gradient of ffn_route_gather.
 */
int ffn_route_combine(const void *ys, const int32_t *place, const float *weights, void *y, int64_t ldy, int64_t N,
                      int32_t per_row, int64_t width, int32_t dtype, void *hip_stream);

/*
 * Gradients of sum(grad_y * y) for ffn_route_combine, grad_y with row stride ldg:
 *   grad_ys [S, width]: weights[n, k] * grad_y[n] in row place[n, k]; zeros from offsets[experts] on
 *   grad_weights [N, per_row], 32-bit floats: the product of grad_y[n] with ys[place[n, k]]; 0 without an expert
 * Either may be NULL, not both; ys is read for grad_weights alone, weights (NULL:
 * ones) for grad_ys alone.
 */
int ffn_route_combine_backward(const void *ys, const int32_t *place, const int32_t *offsets, const float *weights,
                               const void *grad_y, int64_t ldg, void *grad_ys, float *grad_weights, int64_t N,
                               int32_t per_row, int32_t experts, int64_t width, int32_t dtype, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* EXPERTS_H */
