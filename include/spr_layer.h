/*
 * spr_layer.h -- token-wise operations of a Llama3-style decoder layer, so
 * that a whole layer can run through the three-phase schedule (paper
 * Sec. 3.1: everything outside attention acts on each token on its own;
 * App. A.6: the weight gradients are the prefix part once plus the suffix
 * parts).  The projection GEMMs are left to the BLAS library.
 *
 * All tensors are bf16 where a call has no dtype argument, row-major, device
 * memory owned by the caller, 16-byte aligned; statistics are fp32.  Rows are
 * tokens.  Calls are asynchronous on `stream`; on a validation error nothing is launched and
 * spr_last_error() says why.
 */
#ifndef SPR_LAYER_H
#define SPR_LAYER_H

#include "spr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* RMSNorm with unit gain: y = x * r, r = 1 / sqrt(mean(x^2) + eps) per row.
 * x, y [rows, width] (width a multiple of 8, at most 16384); rstd [rows]
 * fp32 out (kept for the backward). */
spr_status spr_rmsnorm_fwd(int32_t rows, int32_t width, float eps, const void* x, void* y,
                           float* rstd, hipStream_t stream);

/* dx = r (dy - x r^2 mean(dy * x)) + add, with r from the forward; `add`
 * [rows, width] (the residual branch's gradient) may be NULL. */
spr_status spr_rmsnorm_bwd(int32_t rows, int32_t width, const void* x, const float* rstd,
                           const void* dy, const void* add, void* dx, hipStream_t stream);

/* Rotary position embedding, rotate-half pairing (j, j + d/2) at angle
 * (pos0 + t) * theta^(-2j/d) for token t: x, y [tokens, heads, head_dim]
 * (head_dim even, at most 256).  The backward is the rotation by the
 * negative angle (inverse = transpose).  Angles are reduced in fp64. */
spr_status spr_rope_fwd(int32_t tokens, int32_t heads, int32_t head_dim, int32_t pos0, double theta,
                        const void* x, void* y, hipStream_t stream);
spr_status spr_rope_bwd(int32_t tokens, int32_t heads, int32_t head_dim, int32_t pos0, double theta,
                        const void* dy, void* dx, hipStream_t stream);

/* RMSNorm of every query and key head with a gain, and the rotary embedding,
 * in one pass (layers that normalise their heads before attention):
 *   z = x g / sqrt(mean(x^2) + eps) over the head's d values (summed in fp32),
 *   y = R z,
 * with R the rotation of spr_rope_fwd at position pos0 + positions[t]
 * (positions: DEVICE int32 [tokens], any values), or pos0 + t where
 * `positions` is NULL.  Packed suffixes, which all start behind one prefix,
 * pass positions.  Unlike the other calls of this header it takes `dtype`
 * SPR_BF16 or SPR_F32 for every tensor but the gain gradients.
 * * q [tokens, q_heads, d], k [tokens, kv_heads, d]: d contiguous, heads d
 *   apart, tokens q_stride / k_stride elements apart (at least a token's own
 *   heads, at most 2^31 - 1), so both may be views of one fused projection;
 *   any element alignment, 16 bytes (and strides of as much, d a multiple of
 *   16) being the fast one.  gain_q, gain_k [d].  yq, yk contiguous, out; they
 *   overlap nothing.  tokens * (q_heads + kv_heads), and a token's elements,
 *   are at most 2^31 - 1. */
spr_status spr_head_norm_rope_fwd(int32_t dtype, int32_t tokens, int32_t q_heads, int32_t kv_heads,
                                  int32_t head_dim, float eps, int32_t pos0, const int32_t* positions,
                                  double theta, const void* q, int64_t q_stride, const void* k,
                                  int64_t k_stride, const void* gain_q, const void* gain_k, void* yq,
                                  void* yk, hipStream_t stream);

/* Its backward, from the forward's inputs and dyq, dyk (contiguous): with
 * dz = R^T dy, r the row's 1 / sqrt(mean(x^2) + eps),
 *   dx = r g dz - x r^3 mean(g dz x),   dg = sum over rows of dz x r.
 * dq and dk are written with token strides of their own (views of one fused
 * gradient, say: their rows may interleave, but may not share an element).
 * dgain_q, dgain_k [d] fp32 are written (overwrite != 0) or added to, in a
 * fixed order: bitwise reproducible. */
spr_status spr_head_norm_rope_bwd(int32_t dtype, int32_t tokens, int32_t q_heads, int32_t kv_heads,
                                  int32_t head_dim, float eps, int32_t pos0, const int32_t* positions,
                                  double theta, const void* q, int64_t q_stride, const void* k,
                                  int64_t k_stride, const void* gain_q, const void* gain_k, const void* dyq,
                                  const void* dyk, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride,
                                  float* dgain_q, float* dgain_k, int32_t overwrite, void* ws,
                                  size_t ws_bytes, hipStream_t stream);
spr_status spr_head_norm_rope_bwd_workspace_size(int32_t tokens, int32_t q_heads, int32_t kv_heads,
                                                 int32_t head_dim, size_t* bytes);

/* SwiGLU: m = silu(g) * u; backward dg = dm u silu'(g), du = dm silu(g).
 * All [n] with n a multiple of 8. */
spr_status spr_swiglu_fwd(int64_t n, const void* g, const void* u, void* m, hipStream_t stream);
spr_status spr_swiglu_bwd(int64_t n, const void* g, const void* u, const void* dm, void* dg, void* du,
                          hipStream_t stream);

/* Weight-gradient sums (App. A.6: the prefix part plus every suffix part):
 * dst = src (overwrite != 0) or dst += src, src [n] bf16, dst [n] fp32, n a
 * multiple of 8. */
spr_status spr_grad_accumulate(int64_t n, const void* src, float* dst, int32_t overwrite, hipStream_t stream);

/* Embedding lookup: y[t] = scale * table[ids[t]], y [tokens, width], table
 * [vocab, width], both of `dtype` (SPR_BF16 or SPR_F32); ids DEVICE int32
 * [tokens].  An id outside [0, vocab) (padding) gives a row of zeros.  width a
 * multiple of 8, any vocab >= 1, tokens * width at most 2^39 (here and in the
 * gradient). */
spr_status spr_embed_fwd(int32_t dtype, int32_t tokens, int32_t vocab, int32_t width, float scale,
                         const int32_t* ids, const void* table, void* y, hipStream_t stream);

/* Its gradient, added to an fp32 table (as the prefix's part once plus every
 * suffix's, App. A.6): dtable[v] += scale * sum over t with ids[t] = v of dy[t].
 * Tokens are sorted stably by id and each row is summed in token order by
 * fixed ranges, with no atomics on values: bitwise reproducible.  Ids outside
 * [0, vocab) are skipped; rows of ids that do not occur are not touched. */
spr_status spr_embed_bwd(int32_t dtype, int32_t tokens, int32_t vocab, int32_t width, float scale,
                         const int32_t* ids, const void* dy, float* dtable, void* ws, size_t ws_bytes,
                         hipStream_t stream);
spr_status spr_embed_bwd_workspace_size(int32_t tokens, int32_t vocab, int32_t width, size_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* SPR_LAYER_H */
