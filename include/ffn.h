/*
 * ffn.h: C ABI of the feed-forward sublayer that networks place around the
 * tensor products, on MI355X (gfx950): the gated feed-forward block (the
 * network that makes per-pair path weights for cgtp_forward_weighted, or mixes
 * scalar channels), the norms before and after a block fused with its gate and
 * residual scale, the layer norm, and dropout from a counter-based generator.
 * Each has its gradients.
 *
 * Arrays are row-major device arrays of one type:
 *   FFN_FP32, FFN_BF16 or FFN_FP16.
 * Sums, statistics and the arithmetic between a read and a write are held in
 * 32 bits; what is stored is rounded to the arrays' type once, to nearest.
 *
 * Row strides (ldx, ...) count elements and must be >= the row's width; the
 * elements of a row are adjacent.  Arrays that have a row stride, and those of
 * the norms and of dropout, need the alignment of their element; the weights
 * and results of ffn_forward and ffn_backward start on 16 bytes
 * (CGTP_EINVAL).  No output may overlap an input, the workspace or another
 * output (CGTP_EINVAL), except where a call says so; neighbouring columns of one
 * array (rows of one stride that share no element) do not overlap.
 *
 * Every call runs asynchronously on hip_stream (NULL: the default stream) of
 * the current device, which must be the arrays' own, allocates nothing, and may
 * be captured in a HIP graph; scratch memory is the caller's workspace,
 * 256-byte aligned, of the size that the matching query gives, whose contents
 * need not be kept between calls.  N == 0 returns CGTP_OK; gradients that sum
 * over rows are then zero.  Status codes are those of cgtp.h, and
 * cgtp_strerror / cgtp_last_hip_error apply.
 */
#ifndef FFN_H
#define FFN_H

#include <stdint.h>

#include "cgtp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FFN_FP32 = 0, FFN_BF16 = 2, FFN_FP16 = 3 }; /* FFN_FP32 == CGTP_FP32 */

/* silu(g) = g / (1 + exp(-g)); gelu(g) = g (1 + erf(g / sqrt 2)) / 2; relu(g) = max(g, 0) */
enum { FFN_SILU = 0, FFN_GELU = 1, FFN_RELU = 2 };

/* Largest d_in, d_ff, d_out and norm width; largest N of one call. */
#define FFN_MAX_WIDTH (1LL << 20)
#define FFN_MAX_ROWS (1LL << 30)

/* ------------------------------------------------------------------ gated feed-forward block
 *
 *   G = X Wg^T,  U = X Wu^T,  H = act(G) * U,  Y = H Wo^T
 *
 *   X     [N, d_in], row stride ldx
 *   w_in  [2 d_ff, d_in]: the d_ff rows of Wg, then the d_ff rows of Wu
 *   w_out [d_out, d_ff] = Wo
 *   Y     [N, d_out]
 * Both projections are one product, with the activation and the product with U
 * in its epilogue: G and U are written only where `saved` asks for them
 * (training).  Where that product is cut along d_in, having few tiles, its parts'
 * 32-bit sums pass through the workspace and a second kernel finishes them.
 */
typedef struct ffn_plan_s *ffn_plan_t;

/*
 * A plan for blocks of one shape on the current HIP device; it owns no device
 * memory.  CGTP_EINVAL for a size below 1, an unknown activation or plan_out
 * NULL; CGTP_EUNSUP for a size above FFN_MAX_WIDTH; CGTP_EDTYPE; CGTP_ENOMEM;
 * CGTP_EHIP.  *plan_out is written only on success.
 */
int ffn_plan(int64_t d_in, int64_t d_ff, int64_t d_out, int32_t activation, int32_t dtype, ffn_plan_t *plan_out);

/* Frees the plan.  NULL is a no-op. */
int ffn_destroy(ffn_plan_t plan);

/* Workspace bytes ffn_forward needs for N rows (the same with and without `saved`); -1 for a NULL plan or N out of range. */
int64_t ffn_workspace_bytes(ffn_plan_t plan, int64_t N);

/* Workspace bytes ffn_backward needs for N rows; -1 as above. */
int64_t ffn_backward_workspace_bytes(ffn_plan_t plan, int64_t N);

/*
 * Y of N rows.  saved: NULL, or [N, 2 d_ff] 32-bit floats, whatever the
 * arrays' type, to receive G (the first d_ff columns) and U of every row for
 * ffn_backward (rounded to 16 bits they would double the error of every
 * gradient).  CGTP_EINVAL for NULL or
 * misaligned arrays, N < 0, ldx < d_in, overlaps, a workspace that is too
 * small, or another current device than the plan's; CGTP_EUNSUP for
 * N > FFN_MAX_ROWS, ldx > 2^21, or products of more than 2^22 tiles of
 * 128 x 128 (256 x 256 where those are faster).
 *
 * H is held in the arrays' type between the two products (as dG, dU and H are
 * in ffn_backward): in fp16 its values above 65504 become infinite.  32-bit
 * products of more than 64 rows, and the weights' gradients, run as six products
 * of bf16 parts of the operands, added in 32 bits: beside the rounding of the
 * sum, each product x w is off by at most 2^-22 |x w|, of either sign (2^-25.5 in
 * the root mean square; a 32-bit product is off by up to 2^-24); there a value
 * that is not finite gives NaN in every sum that it enters.
 */
int ffn_forward(ffn_plan_t plan, const void *x, int64_t ldx, const void *w_in, const void *w_out, void *y,
                void *saved, int64_t N, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * Gradients of sum(grad_y * Y):
 *   dH = dY Wo,  dU = dH * act(G),  dG = dH * U * act'(G)   (relu'(0) = 0)
 *   grad_x [N, d_in]        = [dG dU] w_in
 *   grad_w_in [2 d_ff, d_in] = [dG dU]^T X
 *   grad_w_out [d_out, d_ff] = dY^T H
 * saved is what ffn_forward wrote; grad_y [N, d_out] has row stride ldg.  Any
 * of the three gradients may be NULL (not computed), not all.  Otherwise as
 * ffn_forward.
 */
int ffn_backward(ffn_plan_t plan, const void *x, int64_t ldx, const void *w_in, const void *w_out, const void *saved,
                 const void *grad_y, int64_t ldg, void *grad_x, void *grad_w_in, void *grad_w_out, int64_t N,
                 void *workspace, int64_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------ norms, gate, residual scale
 *
 *   N(v; w) = v / sqrt(mean(v^2) + eps) * w            over the `width` values of a row
 *   before a block:  u = N(x; w)
 *   after a block:   y = x + scale * gate * drop(N(h; w)),  and, in the same pass,
 *                    u = N(y; w_next), the norm before the next block
 * gate is [ceil(N / rows_per_gate), width]: row r takes gate row
 * r / rows_per_gate (rows_per_gate consecutive rows share one, the last ones
 * possibly fewer); scale, w and w_next are [width].  drop is the dropout below
 * with counter row r.
 */
typedef struct {
    int64_t width;         /* 1 .. FFN_MAX_WIDTH */
    int64_t rows_per_gate; /* >= 1; read where a gate is given */
    int32_t dtype;         /* FFN_FP32, FFN_BF16, FFN_FP16 */
    float eps;             /* > 0, finite */
    double dropout;        /* 0 .. 1: probability of dropping (0: none) */
    uint64_t seed;         /* the generator's key and the upper half of its counter, see ffn_dropout */
    uint64_t offset;
} ffn_norm;

/*
 * u = N(x; w) of N rows; x and u have row strides ldx and ldu.  w NULL: all
 * ones.  rstd: NULL, or [N] floats to receive 1 / sqrt(mean + eps).  u == x
 * with ldu == ldx is allowed.  CGTP_EINVAL, CGTP_EDTYPE, CGTP_EUNSUP as for
 * ffn_forward.
 */
int ffn_norm_forward(const ffn_norm *norm, const void *x, int64_t ldx, const void *w, void *u, int64_t ldu,
                     float *rstd, int64_t N, void *hip_stream);

/*
 * Gradients of sum(grad_u * N(x; w)): grad_x [N, width] and grad_w [width]
 * (either may be NULL, not both).  rstd is what ffn_norm_forward wrote;
 * grad_u has row stride ldg.  Workspace: ffn_norm_workspace_bytes(norm, N, 0).
 */
int ffn_norm_backward(const ffn_norm *norm, const void *x, int64_t ldx, const void *w, const float *rstd,
                      const void *grad_u, int64_t ldg, void *grad_x, void *grad_w, int64_t N, void *workspace,
                      int64_t workspace_bytes, void *hip_stream);

/*
 * y (and u) of N rows.  x, h, y, u: [N, width], contiguous.  gate, scale and
 * w NULL: ones.  u NULL: no next norm (w_next is then not read); u given and
 * w_next NULL: ones.  stats: NULL, or [2, N] floats to receive 1 / sqrt(mean +
 * eps) of h's rows and, where u is given, of y's.  y == x is allowed.
 */
int ffn_residual_forward(const ffn_norm *norm, const void *x, const void *h, const void *w, const void *gate,
                         const void *scale, const void *w_next, void *y, void *u, float *stats, int64_t N,
                         void *hip_stream);

/*
 * Gradients of sum(grad_y * y) + sum(grad_u * u) for ffn_residual_forward
 * with the same norm, gate, scale, w and w_next (h and y are read, x is not).
 * grad_y or grad_u may be NULL (zero), not both; grad_u needs y and stats of
 * y's rows.  Outputs, each NULL where it is not wanted: grad_x, grad_h
 * [N, width]; grad_w, grad_scale, grad_w_next [width]; grad_gate like gate.
 * grad_x and grad_h are required; grad_x == grad_y is allowed.  grad_w_next
 * is zero where grad_u is NULL.  Workspace:
 * ffn_norm_workspace_bytes(norm, N, 1).
 */
int ffn_residual_backward(const ffn_norm *norm, const void *h, const void *y, const void *w, const void *gate,
                          const void *scale, const void *w_next, const float *stats, const void *grad_y,
                          const void *grad_u, void *grad_x, void *grad_h, void *grad_w, void *grad_gate,
                          void *grad_scale, void *grad_w_next, int64_t N, void *workspace, int64_t workspace_bytes,
                          void *hip_stream);

/* Workspace bytes of ffn_norm_backward (residual = 0) or ffn_residual_backward (residual = 1); -1 if invalid. */
int64_t ffn_norm_workspace_bytes(const ffn_norm *norm, int64_t N, int32_t residual);

/* ------------------------------------------------------------------ layer norm
 *
 *   L(x; w, b) = (x - m) r * w + b,  m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps)
 * over the `width` values of a row, for scalar features that carry an offset.
 * Of the description, width, dtype and eps are read (the rest has to be valid).
 */

/*
 * u = L(x; w, b) of N rows; x and u have row strides ldx and ldu.  w NULL: all
 * ones; b NULL: zeros.  stats: NULL, or [2, N] floats to receive m and then r of
 * the rows.  u == x with ldu == ldx is allowed.  A row whose mean square deviation
 * passes the range of 32 bits has r = 0.  Statuses as ffn_norm_forward.
 */
int ffn_layer_forward(const ffn_norm *norm, const void *x, int64_t ldx, const void *w, const void *b, void *u,
                      int64_t ldu, float *stats, int64_t N, void *hip_stream);

/*
 * Gradients of sum(grad_u * L(x; w, b)): with n = (x - m) r and a = grad_u w,
 *   grad_x [N, width] = r (a - mean(a) - n mean(a n)),
 *   grad_w [width] = sum over rows of grad_u n,  grad_b [width] = that of grad_u;
 * any of them may be NULL, not all.  stats is what ffn_layer_forward wrote; m is
 * corrected for its rounding.  grad_u has row stride ldg.  Workspace:
 * ffn_layer_workspace_bytes(norm, N).
 */
int ffn_layer_backward(const ffn_norm *norm, const void *x, int64_t ldx, const void *w, const float *stats,
                       const void *grad_u, int64_t ldg, void *grad_x, void *grad_w, void *grad_b, int64_t N,
                       void *workspace, int64_t workspace_bytes, void *hip_stream);

/* Workspace bytes of ffn_layer_backward; -1 if invalid. */
int64_t ffn_layer_workspace_bytes(const ffn_norm *norm, int64_t N);

/* ------------------------------------------------------------------ dropout
 *
 * y[r, c] = x[r, c] * 65536 / (65536 - t) where draw(r, c) >= t, else 0, with
 * t = floor(65536 p + 1/2), for r < N, c < width.  t = 65536 drops everything.
 * draw is a whole number of 16 bits that depends on (seed, offset, r, c)
 * alone: Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw,
 * "Parallel random numbers: as easy as 1, 2, 3", SC 2011) at counter
 * (c / 8, r, low half of offset, high half of offset) and key (low half of
 * seed, high half of seed) gives 128 bits, words in order, low halves first;
 * column c takes the (c mod 8)-th 16 of them.  The mask is never stored: the
 * gradient of y with respect to x is the same call on the gradient.  Dropped
 * values are zero also where x is not finite.  Two calls are independent
 * where seed or offset differ.
 * x and y have row strides ldx and ldy; y == x with ldy == ldx is allowed.
 * CGTP_EINVAL for p outside [0, 1] or not a number.
 */
int ffn_dropout(const void *x, int64_t ldx, void *y, int64_t ldy, int64_t N, int64_t width, int32_t dtype, double p,
                uint64_t seed, uint64_t offset, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* FFN_H */
