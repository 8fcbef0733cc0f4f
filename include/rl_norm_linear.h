/*
 * rl_norm_linear.h - C ABI of the layers in front of the LM head: layer norm, 8-bit checkpoints, 8-bit linear layer (MI355X / gfx950).
 *
 * The final layer norm and a projection y = x W^T stand between a model's last block and the LM head of rl_policy.h; both are trained with it,
 * and what their forward pass keeps for the backward pass is as large as the hidden states themselves.  Here the kept activations, and the operands of the projection,
 * are 8-bit rows:
 *     codes  [rows, rl_f8_code_pitch(K)]   one byte a value, e4m3 (OCP, no infinities) or e5m2; K rounded up to 128, pads zero
 *     scales [rows, rl_f8_scale_pitch(K)]  one byte s for 128 consecutive values of a row, their factor being 2^(s - 127)
 * with the smallest scale under which the largest finite magnitude of the 128 values is representable (448 or 57344; byte 127 for zeros only; at least
 * 2^-127).  Values are rounded to nearest even (one that this would put beyond f32's largest, to the largest below it); infinities (e5m2 keeps them) and NaN become NaN and set no scale.  A weight has one scale for 128 x 128 values, written
 * for each of its rows, so that W and its transpose hold the same values.
 *
 * Conventions are those of rl_policy.h: device pointers owned by the caller, nothing allocated, kept or synchronised, all work on `stream`, host-checkable errors
 * returned before anything is launched, results the same bits every run.  x, y, dy, dx are [rows, columns] with a row stride (ld*) of
 * at least the columns, in elements, and need no more alignment than an element; codes, scales and f32 outputs of this header 16 bytes; workspaces 256.
 * Rows may be 0: outputs without rows are left alone, gradients of parameters are zero.  RL_ERR_DTYPE: unknown rl_dtype or rl_f8_format.
 */
#ifndef RL_NORM_LINEAR_H
#define RL_NORM_LINEAR_H

#include "rl_policy.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum rl_f8_format { RL_E4M3 = 0, RL_E5M2 = 1 } rl_f8_format;

#define RL_LAYER_NORM_MAX_H 16384

/* Host only: bytes of a row of codes / of scales for K columns. */
int64_t rl_f8_code_pitch(int32_t K);
int64_t rl_f8_scale_pitch(int32_t K);

/* y = (x - mean) rstd gamma + beta over the H columns of each row, mean and rstd = (var + eps)^(-1/2) (population variance) in f32.
 *   x, y [R, H] in `dtype`; y may be x, with the same stride;  gamma, beta [H] in `param_dtype`, beta may be NULL (none);  H at most RL_LAYER_NORM_MAX_H;
 *   eps finite and >= 0;  stats [R, 2] f32: mean and rstd for the backward pass, or NULL;
 *   codes, scales: an 8-bit checkpoint of x in `format`, or both NULL (format is then not looked at). */
rl_status rl_layer_norm_forward(const void* x, int64_t ldx, int32_t dtype, int64_t R, int32_t H, const void* gamma, const void* beta,
                                int32_t param_dtype, float eps, void* y, int64_t ldy, float* stats, void* codes, void* scales,
                                int32_t format, void* stream);

/* dx, dgamma [H] and dbeta [H] (f32, overwritten; dbeta may be NULL) from dy and either x or its checkpoint (x NULL, codes and scales given), with the
 * statistics of the forward pass.  dx may be dy, or x, with the same stride.  A row whose dy is zero contributes nothing and gets dx = 0, whatever its x holds. */
rl_status rl_layer_norm_backward_workspace_bytes(int64_t R, int32_t H, size_t* bytes);
rl_status rl_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* codes, const void* scales, int32_t format,
                                 int32_t dtype, int64_t R, int32_t H, const void* gamma, int32_t param_dtype, const float* stats,
                                 void* dx, int64_t lddx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream);

/* x [R, K] to 8-bit rows, and back (exact in f32; rounded where bf16 cannot hold it, which only values below its normal range need). */
rl_status rl_f8_pack(const void* x, int64_t ldx, int32_t dtype, int64_t R, int32_t K, int32_t format, void* codes, void* scales, void* stream);
rl_status rl_f8_unpack(const void* codes, const void* scales, int32_t format, int64_t R, int32_t K, void* x, int64_t ldx, int32_t dtype, void* stream);

/* W [N, K] to 8-bit rows, one scale for 128 x 128 values; codes_t, scales_t: the transpose [K, N] as well (the operand of dx), or both NULL. */
rl_status rl_f8_pack_weight(const void* w, int64_t ldw, int32_t dtype, int32_t N, int32_t K, int32_t format, void* codes, void* scales,
                            void* codes_t, void* scales_t, void* stream);

/* y [M, N] = x w^T of two matrices of 8-bit rows with K columns, x [M, K] and w [N, K]; y in `dtype`.  y in f32: exact
 * products, added in f32 (values taken to 2^-133, where bf16 ends).  y in bf16: the matrix unit adds eight products at a time on a common exponent, what is below 2^-13 of the largest of the eight being cut off,
 * and those sums in f32; together at most 2^-10 of the sum of the products' magnitudes, in the mean a hundredth of y's own rounding.  The linear layer's y and dx likewise. */
rl_status rl_f8_matmul_workspace_bytes(int64_t M, int32_t N, int32_t K, size_t* bytes);
rl_status rl_f8_matmul(const void* x_codes, const void* x_scales, int32_t x_format, const void* w_codes, const void* w_scales, int32_t w_format,
                       int64_t M, int32_t N, int32_t K, void* y, int64_t ldy, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream);

/* The linear layer.  Forward: x [M, K] is packed into x_codes, x_scales (the checkpoint of the backward pass; both NULL: not kept) and multiplied with the packed
 * weight; y must not overlap x.  Workspace: with the packed x kept (keep != 0) or not. */
rl_status rl_f8_linear_forward_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t keep, size_t* bytes);
rl_status rl_f8_linear_forward(const void* x, int64_t ldx, int32_t dtype, int64_t M, int32_t K, int32_t x_format, const void* w_codes,
                               const void* w_scales, int32_t w_format, int32_t N, void* y, int64_t ldy, void* x_codes, void* x_scales,
                               void* workspace, size_t workspace_bytes, void* stream);

/* Backward, from dy [M, N]:  dx [M, K] (in `dtype`; NULL: not wanted) = pack(dy) W, with dy packed in dy_format and the packed transpose of W;
 * dW [N, K] f32 (NULL: not wanted), overwritten, or added to if accumulate is not 0, = dy^T x, with dy as it is and x from the checkpoint.
 * Workspace: by the first query enough for any call of these sizes, by the second for the call at hand.  dx and dW must not overlap dy.  A row whose dy is zero contributes nothing to dW, whatever its x holds.
 * (f32 dy: taken to 2^-24 of each value, or to 2^-133 if that is more; bf16 dy: where it holds infinities or NaN the rows of dW concerned are not finite, which of the two they hold is not specified.) */
rl_status rl_f8_linear_backward_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t dtype, size_t* bytes);
/* What one call needs, at most that: dy_aligned: dy lies on 16 bytes (bf16 rows that all do are not copied); want_dx, want_dW: the output is not NULL. */
rl_status rl_f8_linear_backward_workspace_bytes_for(int64_t M, int32_t N, int32_t K, int32_t dtype, int64_t lddy, int32_t dy_aligned, int32_t want_dx,
                                                    int32_t want_dW, size_t* bytes);
rl_status rl_f8_linear_backward(const void* dy, int64_t lddy, int32_t dtype, int64_t M, int32_t N, int32_t K, int32_t dy_format,
                                const void* x_codes, const void* x_scales, int32_t x_format, const void* wt_codes, const void* wt_scales, int32_t w_format,
                                void* dx, int64_t lddx, float* dW, int64_t lddw, int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RL_NORM_LINEAR_H */
