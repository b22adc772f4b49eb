/*
 * ffn_group_q.h -- matrix-vector products with 4-bit weights and group scales, for a decode step's
 * tokens (gfx950).
 *
 * The *_q calls of ffn_sparse.h take one scale for a stored row.  Here a row's codes have a scale, and
 * an offset where the codes are not symmetric, for every `group` of them along the summed dimension:
 *   W[o][i] = scale[o][i / group] code[o][i] + offset[o][i / group]
 *   ffn_group_q_forward        y = x W^T
 *   ffn_group_q_gated_forward  z = A(x W1^T - t) (*) U(x W3^T), the gated block's hidden layer
 *                              (ffn_gated.h); its way back is a ffn_group_q_forward of z.
 *
 * Codes are two's-complement nibbles, two to a byte, element 2k of a row in the low nibble of the row's
 * byte k (ffn_sparse.h's FFN_I4).  Unsigned codes u with a zero point p, scale (u - p), are code = u - 8
 * (the byte XOR 0x88) and offset = scale (8 - p).
 *
 * Types: x and y are xdt, FFN_BF16 or FFN_F32; scales and offsets are w->sdt, either of the two.
 * Products and sums are fp32: the codes enter the bf16 matrix products as they are (small integers), x as
 * itself, or with FFN_F32 as a sum of three bf16 parts that hold its 24 bits (parts below 2^-122 are flushed);
 * each group's sum is then scaled.  fp32 results are as exact as a plain fp32 sum's, whatever the tokens'
 * signs.  With FFN_BF16 y and z are rounded once.
 *
 * Layouts: row-major device pointers, 16-byte aligned: x [T][n_in], y [T][n_out], codes
 * [n_out][n_in / 2], scales and offsets [n_out][n_in / group].  group is a multiple of 32 and divides
 * n_in.  Any T: tokens go through in passes of 64, each of which reads the weights once.
 *
 * Ownership, streams, errors: as in ffn_sparse.h.  The workspace needs no initialisation, holds nothing
 * from one call to the next, and serves calls of fewer tokens too.  Outputs overlap nothing.
 *
 * Determinism: results are bit-reproducible (no atomic adds; shares of a sum are joined in a fixed order).
 * A token's result does not depend on the other tokens, but may in its last bits on their number.
 *
 * Special values: an Inf or NaN of a token makes that token's outputs Inf or NaN, and no other's; one among a row's scales
 * or offsets reaches that row's outputs alone.  A NaN gate value behaves as in ffn_gated.h.  Sums of a group's
 * x of 2^120 and more may overflow.
 */
#ifndef FFN_GROUP_Q_H
#define FFN_GROUP_Q_H

#include "ffn_sparse.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A quantized matrix (host memory, read during the call only).  offsets: NULL for symmetric codes. */
typedef struct {
  const void* codes;
  const void* scales;
  const void* offsets;
  ffn_dtype_t sdt;
  int group;
} ffn_group_q_t;

/* Bytes of workspace for the calls below (gated: 1 for the gated one); 0 for an invalid shape. */
size_t ffn_group_q_workspace_bytes(int T, int n_in, int n_out, int gated);

/* Errors: FFN_ERR_NULL, _SHAPE (T, n_in, n_out < 1; n_in or n_out above 2^20; T n_in, T n_out or n_in n_out
 * of 2^31 and more; group not a positive multiple of 32 or not a divisor of n_in), _DTYPE (xdt, sdt), _ALIGN,
 * _OPTION (opt as for ffn_gated_forward; sdt, group or offsets that differ between the two matrices), _WORKSPACE, _HIP. */
int ffn_group_q_forward(ffn_dtype_t xdt, int T, int n_in, int n_out, const void* x, const ffn_group_q_t* w, void* y,
                        void* ws, size_t ws_bytes, hipStream_t stream);
int ffn_group_q_gated_forward(ffn_dtype_t xdt, int T, int n_in, int n_out, const void* x, const ffn_group_q_t* w_gate,
                              const ffn_group_q_t* w_up, float t, const ffn_options_t* opt, void* z, void* ws,
                              size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FFN_GROUP_Q_H */
