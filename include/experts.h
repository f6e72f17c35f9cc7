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
 * place, source and offsets are device arrays that ffn_route wrote, for as many
 * rows, choices and experts; entries out of their range read and write nothing out
 * of bounds, but give other results.  Of a 16-bit array of the blocks whose rows do
 * not all start on four bytes, the two bytes behind its last value may be read
 * where they are on the same page of memory (4096 bytes); no result depends on them.
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

/* ------------------------------------------------------------------ the experts' gated blocks
 *
 * For the sorted rows p of expert e, X_p being row source[p] / per_row of x:
 *   G = X Wg_e^T,  U = X Wu_e^T,  H = act(G) * U,  Y = H Wo_e^T
 *   w_in  [experts, 2 d_ff, d_in]: of each expert, the d_ff rows of Wg, then those of Wu
 *   w_out [experts, d_out, d_ff]
 * How many rows an expert has is known on the device alone: nothing is copied to the host.
 */
typedef struct ffn_experts_s *ffn_experts_t;

/*
 * A plan on the current HIP device, as ffn_plan makes one for a single block; it
 * owns no device memory.  CGTP_EUNSUP also for experts above FFN_MAX_EXPERTS, or
 * weights of more than 2^30 rows (experts * 2 d_ff, experts * d_out).
 */
int ffn_experts_plan(int32_t experts, int64_t d_in, int64_t d_ff, int64_t d_out, int32_t activation, int32_t dtype,
                     ffn_experts_t *plan_out);

/* Frees the plan.  NULL is a no-op. */
int ffn_experts_destroy(ffn_experts_t plan);

/* Workspace bytes ffn_experts_forward (ffn_experts_backward) needs; -1 for a NULL plan, N or per_row out of range. */
int64_t ffn_experts_workspace_bytes(ffn_experts_t plan, int64_t N, int32_t per_row);
int64_t ffn_experts_backward_workspace_bytes(ffn_experts_t plan, int64_t N, int32_t per_row);

/*
 * y [S, d_out] of the sorted rows; rows from offsets[experts] on are left as they
 * were.  x: [N, d_in], row stride ldx.  saved: NULL, or [S, 2 d_ff] 32-bit floats
 * to receive G and U of the sorted rows for ffn_experts_backward.  Roundings and
 * statuses as ffn_forward.
 */
int ffn_experts_forward(ffn_experts_t plan, const void *x, int64_t ldx, const int32_t *place, const int32_t *source,
                        const int32_t *offsets, const void *w_in, const void *w_out, void *y, void *saved, int64_t N,
                        int32_t per_row, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * Gradients of sum(grad_y * y), grad_y [S, d_out] in the sorted order (rows from
 * offsets[experts] on are not read):
 *   grad_x [N, d_in]: of each row the sum over its choices, added in 32 bits (zeros where it has none)
 *   grad_w_in, grad_w_out like the weights (zeros for an expert without rows)
 * Any may be NULL, not all.  saved is what ffn_experts_forward wrote.
 */
int ffn_experts_backward(ffn_experts_t plan, const void *x, int64_t ldx, const int32_t *place, const int32_t *source,
                         const int32_t *offsets, const void *w_in, const void *w_out, const void *saved,
                         const void *grad_y, void *grad_x, void *grad_w_in, void *grad_w_out, int64_t N,
                         int32_t per_row, void *workspace, int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* EXPERTS_H */
