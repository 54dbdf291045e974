/*
 * spr_experts.h -- the experts of a mixture-of-experts layer: the plan that
 * sorts a router's choices by expert, the products grouped by expert with
 * ragged sizes (forward, gradient of the rows, gradient of the weights), and
 * the weighted sum that brings the experts' rows back to their tokens.  Part
 * of libspr; spr_moe.h accounts for the same router's auxiliary loss.
 *
 * Everything here acts on each token on its own (paper Sec. 3.1), so a layer
 * of experts runs through the three-phase schedule like a dense one: the
 * prefix's tokens once, then each suffix microbatch's, with the weight
 * gradients the prefix part once plus the suffix parts (App. A.6).
 *
 * A layer, forward (T tokens, k choices a token, R = T k rows):
 *   spr_experts_plan          experts [T, k] -> offsets [E + 1], row_token [R],
 *                             pos [T, k]
 *   spr_experts_fwd           gate and up products of the gathered token rows
 *   spr_swiglu_fwd            on the sorted rows
 *   spr_experts_fwd           down product of the sorted rows
 *   spr_experts_combine_fwd   out_t = add_t + sum_j weights[t,j] y[pos[t,j]]
 * and backward: spr_experts_combine_bwd (dy, dweights), spr_experts_bwd_w and
 * spr_experts_bwd_x of the down product, spr_swiglu_bwd, spr_experts_bwd_w and
 * _bwd_x of gate and up (both at once), and spr_experts_combine_fwd without
 * weights, which adds up each token's k rows.
 *
 * Conventions: 1 <= n_experts <= 1024; 1 <= top_k <= n_experts; n_tokens *
 * top_k <= 2^31 - 1; the products take at most 2^31 - 1025 rows, and widths of
 * as much.  Tensors are bf16, the router's weights, their gradients
 * and the weight gradients fp32, all sums fp32.  Row-major, contiguous, device
 * memory owned by the caller, 16-byte aligned (int32 and the router's fp32
 * arrays: 4-byte).  Outputs overlap nothing unless a call says so.
 * `offsets` and `row_token` are read on the device: offsets are clamped into
 * [0, rows] and each raised to the largest one before it, tokens clamped into
 * [0, x_rows), so that wrong values give wrong rows but no access outside the
 * caller's buffers, and no row to two experts.  Calls
 * are asynchronous on `stream`; on a validation error nothing is launched and
 * spr_last_error() says why.  Every result is bitwise reproducible.
 */
#ifndef SPR_EXPERTS_H
#define SPR_EXPERTS_H

#include "spr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Stable sort of the choices by expert.  experts [n_tokens, top_k] int32.
 * The choices of expert e become rows offsets[e] .. offsets[e + 1] - 1, in
 * (token, j) order; row r is of token row_token[r], and choice (t, j) is row
 * pos[t, j].  A choice outside [0, n_experts) (padding, a dropped token) is no
 * row: its pos is -1, and the row_token of the rows that are then left over,
 * behind offsets[n_experts], are -1.  The same expert twice for one token
 * gives two rows. */
spr_status spr_experts_plan(int32_t n_experts, int32_t top_k, int32_t n_tokens, const int32_t* experts,
                            int32_t* offsets, int32_t* row_token, int32_t* pos, void* ws, size_t ws_bytes,
                            hipStream_t stream);
spr_status spr_experts_plan_workspace_size(int32_t n_experts, int32_t top_k, int32_t n_tokens,
                                           size_t* bytes);

/* y[r] = x[src(r)] w[e(r)] for the rows r of every expert: w [n_experts,
 * in_width, out_width]; src(r) = row_token[r], x [x_rows, in_width], or r where
 * row_token is NULL (x_rows >= rows then).  y [rows, out_width].  w2, y2: a
 * second product of the same rows (gate and up), or both NULL.  Rows behind
 * offsets[n_experts] are left as they were.  Widths are multiples of 8. */
spr_status spr_experts_fwd(int32_t n_experts, int32_t rows, int32_t in_width, int32_t out_width,
                           const int32_t* offsets, const void* x, int32_t x_rows, const int32_t* row_token,
                           const void* w, void* y, const void* w2, void* y2, hipStream_t stream);

/* dx[r] = dy[r] w[e(r)]^T (+ dy2[r] w2[e(r)]^T, or dy2 and w2 both NULL): dx
 * [rows, in_width] in the sorted rows' order, rounded once. */
spr_status spr_experts_bwd_x(int32_t n_experts, int32_t rows, int32_t in_width, int32_t out_width,
                             const int32_t* offsets, const void* dy, const void* w, const void* dy2,
                             const void* w2, void* dx, hipStream_t stream);

/* dw[e] (+)= sum over the rows r of e of x[src(r)]^T dy[r], fp32 [n_experts,
 * in_width, out_width]; overwrite != 0 writes (zeros for an expert without
 * rows), 0 adds.  dy2, dw2: a second pair, or both NULL. */
spr_status spr_experts_bwd_w(int32_t n_experts, int32_t rows, int32_t in_width, int32_t out_width,
                             const int32_t* offsets, const void* x, int32_t x_rows,
                             const int32_t* row_token, const void* dy, float* dw, const void* dy2,
                             float* dw2, int32_t overwrite, hipStream_t stream);

/* out[t] = add[t] + sum over j of weights[t,j] y[pos[t,j]], the sum in fp32 in
 * the order of j.  y [rows, width]; a pos outside [0, rows) is skipped.
 * weights [n_tokens, top_k] fp32, or NULL for ones; add [n_tokens, width] or
 * NULL (it may be `out` itself).  width a multiple of 8. */
spr_status spr_experts_combine_fwd(int32_t n_tokens, int32_t top_k, int32_t rows, int32_t width,
                                   const void* y, const int32_t* pos, const float* weights,
                                   const void* add, void* out, hipStream_t stream);

/* dy[pos[t,j]] = weights[t,j] dout[t] (weights NULL: ones) and dweights[t,j] =
 * <y[pos[t,j]], dout[t]>, fp32, zero for a skipped pos; y and dweights may both
 * be NULL.  Rows that no pos names are left as they were; two choices may not
 * name one row (a plan's never do). */
spr_status spr_experts_combine_bwd(int32_t n_tokens, int32_t top_k, int32_t rows, int32_t width,
                                   const void* dout, const void* y, const int32_t* pos,
                                   const float* weights, void* dy, float* dweights, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SPR_EXPERTS_H */
