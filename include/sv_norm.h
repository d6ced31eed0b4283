/*
 * sv_norm.h - C ABI of layer norm and its backward pass (MI355X, gfx950; part of libsvlinattn.so).
 *
 * Over each row x of width d of a token tensor [B][H][N][d]:
 *
 *     mean = sum x / d,   rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),   xh = (x - mean) rstd,   y = w xh + b
 *
 * Two uses: the hidden states that sv_tconv_block_step works on (H = 1, d the model's width, one w and b), and the heads of an
 * attention that has no denominator (sv_decay.h), where every head's output is brought to scale by itself, with a w and b
 * of its own if wanted.
 *
 * Gradients, with t = w dy:
 *
 *     dx = rstd (t - sum t / d - xh sum (t xh) / d),   dw = sum over rows of dy xh,   db = sum over rows of dy
 */
#ifndef SV_NORM_H
#define SV_NORM_H

#include "sv_linattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Forward.  x describes X, y describes Y: same B, H, N, d and dtype, strides of their own; here d is any multiple of 8 (SV_BF16)
 * or 4 (SV_F32) up to 8192.  Y may be X if x and y have the same strides.
 *  weight, bias   fp32 [weight_heads][d] device, 16-byte aligned, or NULL (ones, zeros)
 *  weight_heads   1: one row of parameters for all rows; H: head h has row h
 *  mean, rstd     fp32 [B][H][N] device, or both NULL: kept for the backward pass
 *  eps            >= 0 and finite (0 with a row of equal values gives infinities or NaN)
 * Sums are fp32 and two-pass: the row is held on chip between its mean and its variance.  Conventions and errors as in sv_linattn.h;
 * one plain kernel, which may be captured into a HIP graph from the first call on. */
sv_status sv_layernorm(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias,
                       int32_t weight_heads, float eps, void *Y, const sv_tensor_desc *y, float *mean, float *rstd,
                       void *stream);

/* Bytes of device workspace of sv_layernorm_backward for rows [B][H][N][d] and any weight_heads; no preparation needed.  Pure host
 * function; 0 for unsupported sizes. */
size_t sv_layernorm_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d);

/* Backward.  dY (described by dy), mean and rstd as the forward call left them.  dX (described by dx) may be dY if dy and dx have the same
 * strides.  dweight, dbias: fp32 [weight_heads][d], overwritten; each may be NULL (weight_heads says all the same which rows
 * `weight` has).  Partial sums of the parameters' gradients go through `workspace` and are combined in a fixed order (results are
 * bit-reproducible); it may be NULL if both are. */
sv_status sv_layernorm_backward(const void *X, const sv_tensor_desc *x, const void *dY, const sv_tensor_desc *dy,
                                const float *weight, int32_t weight_heads, const float *mean, const float *rstd,
                                void *dX, const sv_tensor_desc *dx, float *dweight, float *dbias,
                                void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SV_NORM_H */
