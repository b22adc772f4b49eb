/*
 * ffn_moe.h -- a whole mixture-of-experts layer for a decode step's tokens (gfx950).
 *
 * The router of the paper's Appendix C and its experts, each the gated block of ffn_gated.h:
 *   l_e = <w_router[e], x>,  s = softmax(l) or sigma(l)
 *   the k experts of largest s_e + bias_e (without a bias: of largest l_e); equal ones: the lower index first
 *   w_j = scale s_{e_j}, divided by the sum of the k chosen s with normalize
 *   y = sum over j of w_j FFN_{e_j}(x),  FFN_e(x) = W2_e (A(W1_e x - t) (*) U(W3_e x))
 * The choice is made in 64 bits.  Its sums over d run in 64 bits in an order that does not depend on the
 * other tokens, so a token's experts do not depend on the batch that it comes in.
 *
 * Or the routing is given: `ids` and `weights` are then inputs.  An id outside [0, experts) is no
 * expert; a token without any gets zeros; an expert named twice for a token counts twice.
 *
 * Types: wdt is FFN_BF16 or FFN_F32 and is the type of x, y, the router's and the experts' weights alike; bias and
 * `weights` are fp32.  Sums are fp32 (the router's: fp64).  With FFN_BF16, A(.) (*) U(.) enters W2's
 * product in two bf16 parts, which hold 16 of its bits, and y is rounded once; y sums the experts in fp32.
 *
 * Layouts: row-major device pointers, 16-byte aligned: x, y [T][d], w_router [experts][d], w_gate, w_up,
 * w_down_t [experts][d_ff][d], ids int32 and weights fp32 [T][k] (4-byte aligned), bias [experts] (4-byte aligned).
 * Any d and d_ff.  bf16 rows of odd length take narrow loads and are several times slower; other rows that are not whole
 * 16-byte chunks are somewhat slower (those of whole 128-byte lines are fastest).
 *
 * Ownership, streams, errors: as in ffn_sparse.h.  The workspace needs no initialisation, holds nothing
 * from one call to the next, and serves calls of fewer tokens too.  Outputs overlap nothing.
 *
 * Determinism: results are bit-reproducible (no floating-point atomic adds).
 *
 * Special values: an Inf or NaN of a token stays in that token's y and weights; its experts are then k different ones
 * with no further meaning.  A NaN score counts as the lowest.  With normalize, chosen scores
 * that are all below what 64 bits hold (logits more than 700 under 0, or under the largest) give NaN weights.  An
 * expert's weights reach the tokens that chose it alone.  A NaN gate value behaves as in ffn_gated.h.
 */
#ifndef FFN_MOE_H
#define FFN_MOE_H

#include "ffn_sparse.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The router of a call (host memory, read during the call only).
 *   experts, k   1 <= k <= experts; k at most 16, experts at most 512
 *   w            [experts][d], or NULL: the routing is given (the fields below must then be zero)
 *   bias         [experts] fp32 or NULL: added to the scores for the choice alone
 *   sigmoid      1: logistic scores; 0: softmax over all experts
 *   normalize    1: the chosen scores are divided by their sum
 *   scale        factor on the weights; finite */
typedef struct {
  int experts, k;
  const void* w;
  const float* bias;
  int sigmoid;
  int normalize;
  float scale;
} ffn_router_t;

/* Bytes of workspace; 0 for an invalid shape. */
size_t ffn_moe_workspace_bytes(ffn_dtype_t wdt, int T, int d, int d_ff, int experts, int k);

/* The layer.  ids and weights: outputs of the router, or with router->w NULL inputs.  opt as for
 * ffn_gated_forward (NULL: the default form).  T at most 256: more tokens than a decode step has are
 * the gated block's, expert by expert.
 * Errors: FFN_ERR_NULL, _SHAPE (T, d, d_ff < 1, T above 256, d or d_ff above 2^20, d_ff d of 2^31 and
 * more, T k d_ff (d_ff rounded up to 32) of 2^29 and more, experts or k outside the bounds above), _DTYPE, _ALIGN, _OPTION (a
 * field of the router or of opt), _WORKSPACE, _HIP. */
int ffn_moe_forward(ffn_dtype_t wdt, int T, int d, int d_ff, const ffn_router_t* router, const void* x,
                    const void* w_gate, const void* w_up, const void* w_down_t, float t, const ffn_options_t* opt,
                    int32_t* ids, float* weights, void* y, void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FFN_MOE_H */
