/*
 * ffn_norm.h -- the norms before and after a block, fused with the block's gate and the residual
 * stream, and their backward pass (gfx950).
 *
 * A layer adds a block's output f to its residual stream x and hands the next block a norm of the
 * sum.  For each token (row of d components), with RMSNorm as in ffn_sparse.h:
 *   u  = RMSNorm(f) (*) post_gain      the norm after the block (post), or u = f
 *   c  = 1, g or sigma(g)              the gate: none, its values, or the logistic function of them
 *   x' = alpha x + c (*) u             x_out, the residual stream behind the block
 *   n  = RMSNorm(x') (*) pre_gain      n_out, the norm before the next block
 *   RMSNorm(v) = v r,  r = 1 / sqrt(mean v^2 + eps)
 *
 * Gradients, for dn = dL/dn and dx_out = dL/dx' through everything else that reads x', with
 * xh = x' r and fh = f r_f (r_f the post norm's r):
 *   G  = dx_out + r (dn pre_gain - xh mean(dn pre_gain xh))      dpre_gain = sum over tokens dn xh
 *   dx = alpha G,  du = c G,  dc = G u (through sigma: times c (1 - c); a gate of one row: summed over tokens)
 *   df = r_f (du post_gain - fh mean(du post_gain fh)), or du    dpost_gain = sum over tokens du fh
 *
 * Types: dt is FFN_BF16 or FFN_F32, the type of every tensor but rstd (fp32).  All arithmetic is
 * fp32; n is computed from x' before x' is rounded, and each output is rounded once.  The backward call
 * reads x' as it was stored.
 *
 * Layouts: row-major device pointers, 16-byte aligned: x, f, x_out, n_out and their gradients
 * [T][d], gains [d], the gate [1][d] or [T][d].  Any d up to 16384; d not a multiple of 8 (bf16) or 4
 * (fp32) takes 16-byte loads too, but for the chunk that a row ends in, and is slower for it.
 *
 * Ownership, streams, errors: as in ffn_sparse.h.  x_out may be x itself, and dx may be
 * dx_out; outputs otherwise overlap nothing.  The backward call's workspace needs no
 * initialisation and holds nothing from one call to the next.
 *
 * Determinism: results are bit-reproducible (no atomic adds; sums over tokens are joined in a fixed
 * order that depends on T and d alone).
 *
 * Range: rows of any finite values are normed, also those whose squares pass fp32's range.  r is fp32: below 2^-126 (rows
 * of more than 2^126) with fewer bits.  Squares below 2^-126 are held to multiples of 2^-149, which only an eps of that size shows.
 *
 * Special values: an Inf or NaN of a token stays in that token's outputs, dx, df and dgate rows; it
 * reaches the gradients that are summed over tokens.
 */
#ifndef FFN_NORM_H
#define FFN_NORM_H

#include "ffn_sparse.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The form of a call (host memory, read during the call only).
 *   alpha         scale of the residual; finite
 *   eps           of both norms; finite and > 0
 *   post          1: the block's output is normed; 0: taken as is
 *   gate_sigmoid  1: the gate is the logistic function of `gate`
 *   gate_rows     rows of `gate`: 0 (no gate, gate NULL), 1 (one for all tokens) or T
 *   post_gain, pre_gain  [d], NULL for ones */
typedef struct {
  float alpha;
  float eps;
  int post;
  int gate_sigmoid;
  int gate_rows;
  const void* gate;
  const void* post_gain;
  const void* pre_gain;
} ffn_norm_t;

/* x_out and n_out from x and the block's output f.  f NULL: the norm before a first block alone
 * (x' = x: alpha 1, no post norm, no gate, x_out NULL; else FFN_ERR_OPTION).  n_out NULL: no norm of x'
 * (pre_gain must be NULL); one of x_out, n_out is given.  rstd: NULL, or [2][T] fp32 (4-byte aligned)
 * for the backward call: r_f of every token (written with post), then r (written with n_out).
 * Errors: FFN_ERR_NULL, _SHAPE (T, d < 1, d above 16384, T d of 2^31 and more), _DTYPE, _ALIGN,
 * _OPTION (a field of the form that is not as above), _HIP. */
int ffn_norm_forward(ffn_dtype_t dt, int T, int d, const void* x, const void* f, const ffn_norm_t* form, void* x_out,
                     void* n_out, float* rstd, hipStream_t stream);

/* Bytes of workspace for ffn_norm_backward (a call of fewer tokens of the same d fits too); 0 for an
 * invalid shape. */
size_t ffn_norm_workspace_bytes(int T, int d);

/* The gradients, from x_out and rstd of the forward call of the same form (with f NULL: x in the place of
 * x_out).  dn NULL: n was not computed or not used; dx_out NULL: x' reaches the loss through n alone; one of
 * them is given.  Each of dx, df, dgate, dpost_gain and dpre_gain may be NULL, and is then not computed
 * (FFN_ERR_NULL if all are; FFN_ERR_OPTION for a gradient of what the form does not have: df without f,
 * dgate without a gate, dpost_gain without post, dpre_gain without dn).  Gradients are written, not
 * accumulated.  rstd is needed with post or dn. */
int ffn_norm_backward(ffn_dtype_t dt, int T, int d, const void* x_out, const void* f, const ffn_norm_t* form,
                      const float* rstd, const void* dn, const void* dx_out, void* dx, void* df, void* dgate,
                      void* dpost_gain, void* dpre_gain, void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FFN_NORM_H */
