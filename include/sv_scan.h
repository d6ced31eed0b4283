/*
 * sv_scan.h - C ABI of the selective state space scan and its backward pass (MI355X, gfx950; part of libsvlinattn.so).
 *
 * Where the decay of sv_decay.h is a constant of its head, here every token chooses, channel by channel, how much of the state it keeps
 * and how much of itself it adds.  Channel c = (head, feature) of a token tensor [B][H][N][d] has a state h of n numbers (n = 8 or 16):
 *
 *     D_t = softplus(dt_t + dt_bias) = log(1 + exp(dt_t + dt_bias))
 *     h_t[i] = exp(D_t A[i]) h_{t-1}[i] + D_t u_t B_t[i]                    i < n
 *     y_t = (sum_i C_t[i] h_t[i] + skip u_t) silu(z_t)                      silu(z) = z / (1 + exp(-z)); without Z: times 1
 *
 * u, dt, z and y are numbers of a channel and token; A, dt_bias and skip belong to a channel; B_t and C_t are n numbers that the H / G
 * heads of a group share, G groups of neighbouring heads (G = 1: all channels share them).
 *
 * Gradients, with y'_t = dy_t silu(z_t) and g_t the gradient of h_t,  g_t = C_t y'_t + exp(D_{t+1} A) g_{t+1}  (dS_out behind the last):
 *
 *     dz_t = dy_t (sum_i C_t[i] h_t[i] + skip u_t) silu'(z_t)      dC_t[i] = sum_c y'_t h_t[i]        dB_t[i] = sum_c g_t[i] D_t u_t
 *     e_t = sum_i g_t[i] B_t[i]      p_t[i] = g_t[i] exp(D_t A[i]) h_{t-1}[i]      dD_t = sum_i A[i] p_t[i] + u_t e_t
 *     du_t = D_t e_t + skip y'_t     ddt_t = dD_t sigmoid(dt_t + dt_bias)          dS_in[i] = exp(D_0 A[i]) g_0[i]
 *     dA[i] = sum_{b, t} D_t p_t[i]  ddt_bias = sum_{b, t} ddt_t                   dskip = sum_{b, t} y'_t u_t
 *
 * Conventions of sv_linattn.h hold: device pointers on the current device, host descriptors, work enqueued on `stream`, no allocation,
 * every argument checked on the host before anything is launched (an error other than SV_ERR_LAUNCH means that nothing was written),
 * bit-reproducible results.  The calls launch plain kernels only and can be captured into a HIP graph from the first call on; two
 * calls that overlap in time need a workspace each.  In addition:
 *  - `u` describes U and DT (and dU, dDT), `z` describes Z (and dZ) and is NULL with it, `y` (`dy`) describes Y (dY): same B, H, N, d
 *    and dtype, strides of their own.  d is any multiple of 8 (SV_BF16) or 4 (SV_F32) up to 8192.
 *  - `bc` describes Bm and Cm (and dB, dC) as [B][G][N][n] of the same dtype: its H is G, a divisor of u's H, its d is n.
 *  - A is fp32 [H][d][n], dt_bias and skip fp32 [H][d], each of the two or NULL (zeros).  A must be numbers and is meant negative (decays); where it is
 *    positive D A of a token must stay below 88 (the range of fp32's exp).  Over a run of tokens a state may grow or decay by any factor, as long as the states, and
 *    what the tokens of any run add to a state of nothing, are in fp32's range themselves; and so for gradients, from the end.
 *  - lengths is int32 [B] or NULL: sequence b has the tokens [0, lengths[b]) of its row (values are held to [0, N]); NULL: N each.  Rows
 *    behind a sequence's last token are neither read nor written.  A sequence of length zero has S_out = S_in.
 *  - States are dense fp32 [B][H][d][n] (in the pool of sv_selective_scan_token [n_slots][H][d][n]).
 *  - Everything is computed in fp32; outputs are rounded once.
 *  - A NaN or an infinity makes what depends on it by the formulas NaN or infinite; outputs of earlier tokens are what they would be
 *    without it, and so are gradients at later ones.
 *  - Outputs must not overlap inputs or each other, but for S_out = S_in and dS_in = dS_out.
 *  - SV_ERR_SHAPE where H d is 2^27 or more, or where a launch would have 2^26 waves or more: one for 64 channels of a group of each sequence, twice as many
 *    backwards (and one for B G N n / 32), n / 4 times as many for single tokens.
 */
#ifndef SV_SCAN_H
#define SV_SCAN_H

#include "sv_linattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device workspace of sv_selective_scan and of sv_selective_scan_backward for these sizes (either dtype; G groups, n numbers of state a channel);
 * contents need no preparation.  What a call needs does for every call with no more batches and tokens and the same H, d, G and n.
 * Backwards it is mostly n + 1 fp32 numbers for every four tokens of a channel: 17 bytes a token and channel at n = 16 (1.25 GB for 32 760 tokens
 * of 2 240 channels).  Every call takes a workspace, a sequence of few tokens that leaves it untouched among them.  Pure host functions; 0 for unsupported arguments. */
size_t sv_selective_scan_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t n);
size_t sv_selective_scan_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t G, int32_t n);

/* Whole sequences (prompts, training).  S_in: the state each sequence begins from, or NULL (zeros).  S_out: receives the state behind
 * its last token, or NULL; may be S_in. */
sv_status sv_selective_scan(const void *U, const void *DT, const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z,
                            const void *Bm, const void *Cm, const sv_tensor_desc *bc, const float *A, const float *dt_bias,
                            const float *skip, const int32_t *lengths, const float *S_in, float *S_out, void *Y,
                            const sv_tensor_desc *y, void *workspace, size_t workspace_bytes, void *stream);

/* One token of each of B sequences (N = 1), states in a pool of n_slots: row b works on slot slots[b] (int32 [B], device; NULL: slot
 * b, then n_slots >= B).  S_out may be S_in (committed in place) or another pool (a step that can be taken back): slots that no row
 * names are left as they are.  A row whose slot is outside [0, n_slots) is idle: nothing of it is read, and its row of Y is left as it
 * is.  A slot named twice serves the first row that names it; the later ones are idle. */
sv_status sv_selective_scan_token(const void *U, const void *DT, const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z,
                                  const void *Bm, const void *Cm, const sv_tensor_desc *bc, const float *A, const float *dt_bias,
                                  const float *skip, const int32_t *slots, int32_t n_slots, const float *S_in, float *S_out, void *Y,
                                  const sv_tensor_desc *y, void *stream);

/* Gradients of sv_selective_scan for all of its inputs.  dY: gradient of Y.  S_in: as given to the forward call.  dS_out: gradient of
 * S_out, or NULL (zeros).  dU, dDT, dZ (NULL without Z), dB and dC are written at the sequences' tokens; dS_in receives the gradient of
 * S_in, or NULL.  dA fp32 [H][d][n], ddt_bias and dskip fp32 [H][d] are overwritten; each may be NULL. */
sv_status sv_selective_scan_backward(const void *U, const void *DT, const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z,
                                     const void *Bm, const void *Cm, const sv_tensor_desc *bc, const void *dY,
                                     const sv_tensor_desc *dy, const float *A, const float *dt_bias, const float *skip,
                                     const int32_t *lengths, const float *S_in, const float *dS_out, void *dU, void *dDT, void *dZ,
                                     void *dB, void *dC, float *dS_in, float *dA, float *ddt_bias, float *dskip, void *workspace,
                                     size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SV_SCAN_H */
