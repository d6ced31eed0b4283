/*
 * sv_norm.h - C ABI of layer norm and group norm and their backward passes (MI355X, gfx950; part of libsvlinattn.so).
 *
 * Layer norm, over each row x of width d of a token tensor [B][H][N][d]:
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
 *
 * Group norm of channels-last hidden states, with an activation: the N rows of a (b, h) - a frame, a clip - share a mean and an rstd in
 * each of G groups of d / G neighbouring channels:
 *
 *     mean = sum x / (N d / G),   rstd = 1 / sqrt(sum (x - mean)^2 / (N d / G) + eps),   xh = (x - mean) rstd,   a = w xh + b
 *     y = a  or  y = silu(a) = a / (1 + exp(-a))
 *
 * Gradients, with da = dy  or  dy silu'(a), and t = w da (means over the rows and channels of a group):
 *
 *     dx = rstd (t - mean of t - xh mean of (t xh)),   dw = sum over all rows of da xh,   db = sum over all rows of da
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

/* Bytes of device workspace of sv_groupnorm and of sv_groupnorm_backward for hidden states [B][H][N][d] in G groups (either dtype); no
 * preparation needed.  What a call needs does for every call with no more batches, heads and rows and the same d and G.  Pure host
 * functions; 0 for unsupported sizes. */
size_t sv_groupnorm_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t groups);
size_t sv_groupnorm_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t groups);

/* Forward.  x describes X, y describes Y: same B, H, N, d and dtype, strides of their own (frames of a clip [B][T][HW][D] are H = T, N =
 * HW: statistics of each frame; H = 1, N = T HW: of the whole clip).  d is any multiple of 8 (SV_BF16) or 4 (SV_F32) up to 8192, groups any
 * divisor of d (groups need not be whole 16-byte pieces).  Y may be X if x and y have the same strides.
 *  weight, bias   fp32 [d] device, 16-byte aligned, or NULL (ones, zeros)
 *  silu           0 or 1
 *  mean, rstd     fp32 [B][H][groups] device, or both NULL: kept for the backward pass
 *  eps            >= 0 and finite (0 with a group of equal values gives infinities or NaN)
 *  workspace      of every call, small ones that leave it untouched among them
 * Refused (SV_ERR_SHAPE) where a launch would have 2^24 workgroups or more: at B H groups + d / 8 or B H (d + 127) / 128 of that many.
 * Sums are fp64.  Conventions and errors as in sv_linattn.h; plain kernels, which may be captured into a HIP graph from the first call on; two calls that overlap in time need a workspace each; results are bit-reproducible. */
sv_status sv_groupnorm(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t groups, float eps,
                       int32_t silu, void *Y, const sv_tensor_desc *y, float *mean, float *rstd, void *workspace,
                       size_t workspace_bytes, void *stream);

/* Backward.  dY (described by dy), mean and rstd as the forward call left them, weight and bias as it had them.  dX (described by dx)
 * may be dY if dy and dx have the same strides.  dweight, dbias: fp32 [d], overwritten; each may be NULL. */
sv_status sv_groupnorm_backward(const void *X, const sv_tensor_desc *x, const void *dY, const sv_tensor_desc *dy, const float *weight,
                                const float *bias, int32_t groups, int32_t silu, const float *mean, const float *rstd, void *dX,
                                const sv_tensor_desc *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes,
                                void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SV_NORM_H */
