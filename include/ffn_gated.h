/*
 * ffn_gated.h -- the gated FFN block over many tokens (prompts, training batches), its backward
 * pass, and low-rank adapters of many requests beside the block's projections (gfx950).
 *
 * The block, tokens in rows (Section 3.1 Eq. (ffn) of the paper that ffn_sparse.h names):
 *   g = x W1^T - t,  v = x W3^T,  z = A(g) (*) U(v),  y = z W2^T
 * with W1 = w_gate, W3 = w_up, W2 stored transposed (w_down_t), A the gate activation of
 * opt->act and U the identity, or SiLU with opt->silu_up.  Every neuron is evaluated: this is
 * the dense form, for many tokens at once and for training a layer (activation casting), where
 * ffn_dense_forward and ffn_sparse_forward take a decode step's tokens.
 *
 * Gradients, for dy = dL/dy:
 *   dz = dy W2,  dg = dz (*) U(v) (*) A'(g),  dv = dz (*) A(g) (*) U'(v)
 *   dx = dg W1 + dv W3,  dW1 = dg^T x,  dW3 = dv^T x,  dW2^T = z^T dy   (all sums over tokens)
 * A' at a border that A is not smooth at (g = 0 for FFN_ACT_RELU and FFN_ACT_RSPLUS) is 0.
 *
 * Adapters: request j has factors A_j [r][in] and B_j [out][r] beside a projection W [out][in];
 * a token with adapter j gets  W x + scale_j B_j (A_j x).
 *
 * Types: wdt is FFN_BF16 or FFN_F32, and is the type of tokens, weights, adapters, outputs and
 * gradients alike (the decode calls' fp32 tokens beside bf16 weights are theirs alone).  Sums are
 * fp32.  With FFN_BF16, z, dg, dv and A_j x are rounded to bf16 where they enter the next matrix
 * product; g and v are kept in fp32 for the backward pass.
 *
 * Layouts: as in ffn_sparse.h (row-major device pointers, 16-byte aligned); x, y, dy, dx
 * [T][d], w_* and dw_* [d_ff][d].  Any d and d_ff; rows that are not whole 16-byte chunks (d not
 * a multiple of 8 bf16 or 4 fp32) are first copied to padded rows in the workspace, so such
 * widths cost a copy of the weights a call.
 *
 * Ownership, streams, errors: as in ffn_sparse.h.  The workspace needs no initialisation,
 * holds nothing from one call to the next, and serves calls of fewer tokens and lower ranks too (its
 * size grows with both).  `save` holds g, v and z of a forward call for the
 * backward call of the same shape and options; it is read only by the backward call, which may
 * be repeated.  Outputs must not overlap inputs, each other, save or the workspace.
 *
 * Determinism: results are bit-reproducible (no atomic adds; shares of a sum are joined in a fixed
 * order).
 *
 * Special values: a NaN gate value gives A = A' = 0 with FFN_ACT_RELU and FFN_ACT_RSPLUS (it is
 * not above the border) and NaN with FFN_ACT_SILU; SiLU of -Inf is NaN too (-Inf times 0).  Inf and
 * NaN of a token reach that token's outputs and dx and every weight gradient, and no other token's; those of an
 * adapter's factors reach the tokens of that adapter only, and g or v only through their own projection.
 */
#ifndef FFN_GATED_H
#define FFN_GATED_H

#include "ffn_sparse.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Adapters of the requests of one call.  n adapters of rank r are held in stacks: a [n][r][in],
 * b [n][out][r].  A projection whose two stacks are NULL has none; both or neither must be given,
 * and at least one projection has some.  in / out: gate and up d / d_ff, down d_ff / d.
 *   ids    [T] int32 (4-byte aligned): the adapter of each token; any value outside [0, n) is none
 *   scale  [n] fp32 (4-byte aligned), or NULL for ones
 * The struct is host memory, read during the call only. */
typedef struct {
  int n, r;
  const int32_t* ids;
  const float* scale;
  const void* gate_a;
  const void* gate_b;
  const void* up_a;
  const void* up_b;
  const void* down_a;
  const void* down_b;
} ffn_adapters_t;

/* Bytes of the buffer that a forward call fills for the backward call; 0 for an invalid shape. */
size_t ffn_gated_save_bytes(ffn_dtype_t wdt, int T, int d_ff);

/* Bytes of workspace for ffn_gated_forward with adapters of rank r (0: none), or, with
 * backward = 1, for both calls.  0 for an invalid shape. */
size_t ffn_gated_workspace_bytes(ffn_dtype_t wdt, int T, int d, int d_ff, int r, int backward);

/* The block.  opt: act FFN_ACT_RELU, FFN_ACT_RSPLUS or FFN_ACT_SILU (all of h - t), silu_up; its
 * other fields are for LoPA gating and must be zero (NULL: the default form).  ad: NULL, or the
 * requests' adapters.  save: NULL, or a buffer of save_bytes >= ffn_gated_save_bytes(...) for the
 * backward call; adapters with save give FFN_ERR_OPTION (the backward call has no adapters).
 * Errors: FFN_ERR_NULL, _SHAPE (T, d, d_ff < 1; d or d_ff above 2^20; d_ff d or T d of 2^31 and
 * more; n or r < 1, r above 2^16, or a stack's r times in or out of 2^31 and more), _DTYPE,
 * _ALIGN, _OPTION, _WORKSPACE (ws_bytes or save_bytes too small), _HIP. */
int ffn_gated_forward(ffn_dtype_t wdt, int T, int d, int d_ff, const void* x, const void* w_gate, const void* w_up,
                      const void* w_down_t, float t, const ffn_options_t* opt, const ffn_adapters_t* ad, void* y,
                      void* save, size_t save_bytes, void* ws, size_t ws_bytes, hipStream_t stream);

/* The gradients, from the save of ffn_gated_forward on the same x, weights, t and options.  dx and
 * each of the dw_* may be NULL, and is then not computed (FFN_ERR_NULL if all are).  Gradients are
 * written, not accumulated.  Needs a workspace of ffn_gated_workspace_bytes(..., backward = 1). */
int ffn_gated_backward(ffn_dtype_t wdt, int T, int d, int d_ff, const void* x, const void* w_gate, const void* w_up,
                       const void* w_down_t, const ffn_options_t* opt, const void* dy, const void* save,
                       size_t save_bytes, void* dx, void* dw_gate, void* dw_up, void* dw_down_t, void* ws,
                       size_t ws_bytes, hipStream_t stream);

/* One shared projection with the requests' adapters: y [T][n_out] = x W^T + scale_j B_j (A_j x),
 * w [n_out][d].  ad's gate_a [n][r][d] and gate_b [n][n_out][r] are its stacks; the others must be
 * NULL (FFN_ERR_OPTION).  Shapes and errors as above, with n_out in the place of d_ff. */
size_t ffn_adapter_workspace_bytes(ffn_dtype_t wdt, int T, int d, int n_out, int r);
int ffn_adapter_forward(ffn_dtype_t wdt, int T, int d, int n_out, const void* x, const void* w,
                        const ffn_adapters_t* ad, void* y, void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FFN_GATED_H */
