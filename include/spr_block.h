/*
 * spr_block.h -- a decoder block outside attention, trained with few bytes of
 * saved activations: the gated feed-forward with its activation in the
 * product's kernel, the norms on both sides of a block with its gate and the
 * scaled residual in one pass, and activations kept in 8 bits, which the first
 * two write as they go and read in their backward.  Part of libspr.
 *
 * Everything here acts on each token on its own (paper Sec. 3.1), so it runs
 * through the three-phase schedule like the layer's other operations; what a
 * layer keeps of its prefix between Phase A and Phase C (Sec. 3.3) is less than
 * half in 8 bits.
 *
 * 8 bits: 32 consecutive values of a row share a scale 2^(e - 127):
 * value = q 2^(e - 127), q int8 [rows, width], e uint8 [rows, ceil(width / 32)]
 * (a row's last block may be shorter).  e is the least at which every |q| is at
 * most 127 after rounding to the nearest (ties to even), and at least 1.  bf16
 * holds such values exactly.  A block with an infinity or a NaN has e = 255 and
 * reads as NaN; magnitudes that round to 2^128 read as infinities, those of up to
 * 2^-127 as zeros.
 *
 * Conventions: tensors are row-major, contiguous, device memory owned by the
 * caller, 16-byte aligned (q: 8-byte; e: any; offsets, row_token and the fp32
 * arrays: 4-byte); widths are multiples of 8; sums and statistics are fp32.
 * Outputs overlap nothing.  Calls are asynchronous on `stream`; on a validation
 * error nothing is launched and spr_last_error() says why.  Every result is
 * bitwise reproducible.
 */
#ifndef SPR_BLOCK_H
#define SPR_BLOCK_H

#include "spr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* x [rows, width] of `dtype` (SPR_BF16 or SPR_F32) to 8 bits.  rows * width at
 * most 2^40. */
spr_status spr_act8_pack(int32_t dtype, int32_t rows, int32_t width, const void* x, int8_t* q, uint8_t* e,
                         hipStream_t stream);

/* y = value (* rstd[row]) (* gain[column]), y and gain [width] of `dtype`, rounded
 * once: the values, or a norm's output formed again from its kept input.  rstd
 * [rows] fp32 and gain may each be NULL. */
spr_status spr_act8_unpack(int32_t dtype, int32_t rows, int32_t width, const int8_t* q, const uint8_t* e,
                           const float* rstd, const void* gain, void* y, hipStream_t stream);

/* The norm after a block, its gate, the residual and the norm before the next
 * block, of a block's output f and its input x:
 *   p = f r_f gain_post      (p = f where rstd_f is NULL)
 *   h = residual_scale x + branch_scale gate p
 *   n = h r_h gain_pre,      r = (mean(row^2) + eps)^-1/2
 * Everything is `dtype` (SPR_BF16 or SPR_F32) [rows, width], width at most
 * 16384.  n, r_h and h's 8 bits are of the fp32 h, which is rounded for h alone.
 * * f NULL: the norm before a first block, n of x; h, rstd_f, gain_post and gate
 *   are NULL then, and h_q takes x.  Without f, rstd_h and n are required.
 * * rstd_f, rstd_h [rows] fp32, out: NULL means no norm on that side (n and
 *   gain_pre, or gain_post, are NULL then).  Gains [width], NULL: ones.
 * * gate: [width], the same for every row, or where gate_per_row is not 0 [rows,
 *   width]; or NULL.
 * * h_q with h_e, f_q with f_e: h and f in 8 bits as well, or NULL. */
spr_status spr_block_norm_fwd(int32_t dtype, int32_t rows, int32_t width, float eps, float residual_scale,
                              float branch_scale, const void* x, const void* f, const void* gain_post,
                              const void* gate, int32_t gate_per_row, const void* gain_pre, void* h, void* n,
                              float* rstd_f, float* rstd_h, int8_t* h_q, uint8_t* h_e, int8_t* f_q,
                              uint8_t* f_e, hipStream_t stream);

/* Its backward, from the kept h and f (of `dtype`, or in 8 bits where h_e, f_e
 * are not NULL), the forward's statistics, and the gradients dh (of h, from the
 * residual stream behind it) and dn (of n), either of which may be NULL:
 *   d  = dh + r_h gain_pre dn - h r_h^3 mean(gain_pre dn h)
 *   dx = residual_scale d,   dp = branch_scale gate d,
 *   df = r_f gain_post dp - f r_f^3 mean(gain_post dp f)   (dp without that norm)
 *   dgain_pre = sum dn h r_h,   dgain_post = sum dp f r_f,
 *   dgate = branch_scale d f r_f gain_post (summed where it is shared)
 * * dn needs h and rstd_h; rstd_f and dgate need f.  dx is required; df, the
 *   gains' gradients and dgate may be NULL.
 * * dgain_pre, dgain_post and a shared gate's dgate are fp32 [width], written where
 *   overwrite is not 0 and added to else, in a fixed order; gates per row
 *   have dgate of `dtype` [rows, width], written. */
spr_status spr_block_norm_bwd(int32_t dtype, int32_t rows, int32_t width, float residual_scale,
                              float branch_scale, const void* h, const uint8_t* h_e, const void* f,
                              const uint8_t* f_e, const float* rstd_f, const float* rstd_h,
                              const void* gain_post, const void* gate, int32_t gate_per_row,
                              const void* gain_pre, const void* dh, const void* dn, void* dx, void* df,
                              float* dgain_post, void* dgate, float* dgain_pre, int32_t overwrite, void* ws,
                              size_t ws_bytes, hipStream_t stream);
spr_status spr_block_norm_bwd_workspace_size(int32_t rows, int32_t width, size_t* bytes);

/* Gated feed-forward, m = act(x w_gate) * (x w_up), for one dense block or for
 * the experts of a layer.  act: SPR_ACT_SILU, or SPR_ACT_GELU_TANH, 0.5 g (1 +
 * tanh(sqrt(2 / pi) (g + 0.044715 g^3))).  bf16; the products, the activation and
 * its product with u are fp32, m is rounded once.
 * * Rows are grouped as in spr_experts.h: offsets [n_experts + 1], row_token
 *   [rows] or NULL; offsets NULL with n_experts 1: all rows.  x [x_rows,
 *   in_width], w_gate, w_up [n_experts, in_width, mid_width], m [rows, mid_width].
 *   Rows behind offsets[n_experts] are left as they were.
 * * g = x w_gate and u = x w_up are kept for the backward where g and u are not
 *   NULL: [rows, mid_width] bf16, or int8 with exponents where g_e and u_e are
 *   not NULL.
 * * Sizes: as spr_experts.h's products, and no more tiles than one launch holds:
 *   about 2^23 of 256 rows of an expert by 128 columns of m (256 in the backward).
 * The down product is spr_experts_fwd, or a BLAS product of a dense block. */
enum { SPR_ACT_SILU = 0, SPR_ACT_GELU_TANH = 1 };
spr_status spr_glu_fwd(int32_t act, int32_t n_experts, int32_t rows, int32_t in_width, int32_t mid_width,
                       const int32_t* offsets, const void* x, int32_t x_rows, const int32_t* row_token,
                       const void* w_gate, const void* w_up, void* m, void* g, uint8_t* g_e, void* u,
                       uint8_t* u_e, hipStream_t stream);

/* Backward through the down product y = m w_down and the activation: with dm =
 * dy w_down^T, formed in fp32 in the kernel,
 *   dg = dm u act'(g),   du = dm act(g),   m = act(g) u,
 * from the kept g and u.  dy [rows, out_width], w_down [n_experts, mid_width,
 * out_width]; dg, du and m [rows, mid_width] (m, which the gradient of w_down
 * needs, may be NULL).  The other gradients are products: dx = spr_experts_bwd_x
 * of dg, w_gate and du, w_up; dw_gate and dw_up = spr_experts_bwd_w of x with dg
 * and du; dw_down = spr_experts_bwd_w of m with dy. */
spr_status spr_glu_bwd(int32_t act, int32_t n_experts, int32_t rows, int32_t mid_width, int32_t out_width,
                       const int32_t* offsets, const void* dy, const void* w_down, const void* g,
                       const uint8_t* g_e, const void* u, const uint8_t* u_e, void* dg, void* du, void* m,
                       hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SPR_BLOCK_H */
