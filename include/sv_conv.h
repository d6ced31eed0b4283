/*
 * sv_conv.h - C ABI of the short causal convolution along tokens and its backward pass (MI355X, gfx950; part of libsvlinattn.so).
 *
 * Each channel c of a token tensor [B][H][N][d] (c = (head, feature)) is mixed with its K - 1 predecessors, K = 2, 3 or 4:
 *
 *     a_t[c] = bias[c] + sum_{j < K} W[j][c] x_{t-(K-1)+j}[c],     y = a  or  y = silu(a) = a / (1 + exp(-a))
 *
 * with x_{-(K-1)} .. x_{-1} = cache_in (zeros without one).  This is what goes before the selective scan of sv_scan.h, or before q, k
 * and v of a decayed attention (sv_decay.h).  The last K - 1 inputs of a sequence, cache and tokens taken together, are cache_out: what
 * the next call goes on from.  (sv_tconv.h mixes whole frames and all channels; here a channel sees itself only.)
 *
 * Gradients, with da = dy  or  dy silu'(a), and da_t = 0 where there is no token t:
 *
 *     dx_t = sum_j W[j] da_{t+(K-1)-j}   (+ dcache_out's row of x_t),   dW[j] = sum_{b, t} da_t x_{t-(K-1)+j},   dbias = sum_{b, t} da_t
 *
 * Conventions of sv_linattn.h hold: device pointers on the current device, host descriptors, work enqueued on `stream`, no allocation,
 * every argument checked on the host before anything is launched (an error other than SV_ERR_LAUNCH means that nothing was written),
 * bit-reproducible results.  The calls launch plain kernels only and can be captured into a HIP graph from the first call on; two
 * calls that overlap in time need a workspace each.  In addition:
 *  - Every tensor has a descriptor of its own; B, H, N, d and dtype agree.  d is any multiple of 8 (SV_BF16) or 4 (SV_F32) up to 8192.
 *  - weight is fp32 [K][H][d], bias fp32 [H][d] or NULL (zeros).
 *  - lengths is int32 [B] or NULL: sequence b has the tokens [0, lengths[b]) of its row (values are held to [0, N]); NULL: N each.  Rows
 *    behind a sequence's last token are neither read nor written.  A sequence of length zero has cache_out = cache_in.
 *  - Caches are dense [B][H][K-1][d] of x's dtype, oldest row first (in the pool of sv_causal_conv_token [n_slots][H][K-1][d]).
 *  - Sums are fp32; outputs and caches are rounded once (caches are copies).
 *  - A NaN or an infinity reaches what depends on it by the formulas and nothing else.
 *  - Outputs must not overlap inputs or each other, but for cache_out = cache_in where that is said.
 *  - SV_ERR_SHAPE where H d is 2^28 or more, or where a launch would have 2^31 threads or more (one for 16 bytes of four to sixteen tokens, backwards for four channels of
 *    eight to 64, 2^24 workgroups at most).
 */
#ifndef SV_CONV_H
#define SV_CONV_H

#include "sv_linattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Whole sequences.  silu: 0 or 1.  cache_in, cache_out: each may be NULL; cache_out may be cache_in. */
sv_status sv_causal_conv(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t taps, int32_t silu,
                         const int32_t *lengths, const void *cache_in, void *cache_out, void *Y, const sv_tensor_desc *y, void *stream);

/* One token of each of B sequences (N = 1), caches in a pool of n_slots: row b works on slot slots[b] (int32 [B], device; NULL: slot
 * b, then n_slots >= B).  cache_out may be cache_in (committed in place) or another pool: slots that no row names are left as they
 * are.  A row whose slot is outside [0, n_slots) is idle: nothing of it is read, and its row of Y is left as it is.  A slot named twice
 * serves the first row that names it; the later ones are idle. */
sv_status sv_causal_conv_token(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t taps, int32_t silu,
                               const int32_t *slots, int32_t n_slots, const void *cache_in, void *cache_out, void *Y,
                               const sv_tensor_desc *y, void *stream);

/* Bytes of device workspace of sv_causal_conv_backward (either dtype, any number of taps); contents need no preparation.  What a call
 * needs does for every call with no more batches, heads and tokens and the same d.  Pure host function; 0 for unsupported sizes. */
size_t sv_causal_conv_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d);

/* Gradients of sv_causal_conv.  dY: gradient of Y.  dcache_out: gradient of cache_out, or NULL (zeros).  dX is written at the sequences'
 * tokens; dcache_in receives the gradient of cache_in, or NULL.  dweight fp32 [K][H][d] and dbias fp32 [H][d] are overwritten; each may
 * be NULL, and the workspace as well if both are. */
sv_status sv_causal_conv_backward(const void *X, const sv_tensor_desc *x, const void *dY, const sv_tensor_desc *dy, const float *weight,
                                  const float *bias, int32_t taps, int32_t silu, const int32_t *lengths, const void *cache_in,
                                  const void *dcache_out, void *dX, const sv_tensor_desc *dx, void *dcache_in, float *dweight,
                                  float *dbias, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SV_CONV_H */
