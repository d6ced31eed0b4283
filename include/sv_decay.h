/*
 * sv_decay.h - C ABI of causal linear attention with a decay for each head (MI355X, gfx950; part of libsvlinattn.so).
 *
 * Beside the block steps of sv_linattn.h, whose attention is full inside a block and whose state never forgets, this is the
 * form that is causal token by token and forgets at a rate of its own in every head.  Per (batch, head), with
 * l = exp(log_decay[h]):
 *
 *     S_t = l S_{t-1} + k_t v_t^T            (d x d, row = key feature, column = value feature, as in sv_linattn.h)
 *     o_t = scale * S_t^T q_t                o_t[v] = scale * sum_k q_t[k] S_t[k][v]
 *
 * that is, o_t = scale * sum_{s <= t} l^{t-s} (q_t . k_s) v_s plus what is left of the state the sequence began from.  q and k
 * are taken as they are: no feature map, no denominator (sv_layernorm of sv_norm.h brings a head's output to scale, sv_rope3d_rotate
 * of sv_rope.h turns q and k before).  A decay is a constant of its head: there is no gradient for it.
 *
 * Conventions of sv_linattn.h hold: device pointers on the current device, host descriptors, work enqueued on `stream`, no
 * allocation, every argument checked on the host before anything is launched (an error other than SV_ERR_LAUNCH means that nothing
 * was written), bit-reproducible results.  The calls launch plain kernels only (no waits inside a kernel, no attributes, no library calls), so
 * they can be captured into a HIP graph from the first call on and replayed with other contents of the same buffers; two calls that
 * overlap in time need a workspace each.  In addition:
 *  - `qkv` describes Q, K and V (and dQ, dK, dV), `o` describes O (and dO): same B, H, N, d and dtype, strides of their own, so that
 *    q, k and v may be views of one projection's output.  64 rows must span less than 2 GiB (else SV_ERR_UNSUPPORTED); heads may
 *    span any number of bytes.
 *  - log_decay is fp32 [H]: 0 keeps everything, minus infinity (l = 0) nothing but the token itself.  Values above 0 grow: a power of l past
 *    the largest fp32 number counts as that number, and results are finite where the formulas' terms are.
 *  - lengths is int32 [B] or NULL: sequence b has the tokens [0, lengths[b]) of its row (values are held to [0, N]); NULL: N each.
 *    Rows behind a sequence's last token are neither read nor written, whatever they hold.  A sequence of length zero has
 *    S_out = S_in.
 *  - SV_BF16: bf16 products with fp32 accumulation; S_out and dS_in are fp32 states (what enters them goes through three bf16 values, 2^-24 of
 *    a term), what comes out of a state on its way to O, dQ, dK and dV and the weighted scores go through pairs of them (2^-16 of a
 *    term), outputs are rounded once.  SV_F32: fp32 products.
 *  - A token's weight l^n in a state many tokens later is an fp32 number: where it has come to zero the token may be passed over.
 *  - A NaN or an infinity in a token, a gradient or a state makes what depends on it by the formulas NaN or infinite, and nothing else: outputs
 *    of earlier tokens are what they would be without it (such a segment is walked twice).  The products q . k of tokens up to 63
 *    apart must stay in the range of fp32, and log decays must be numbers (minus infinity among them).
 *  - Outputs must not overlap inputs or each other, but for S_out = S_in where that is said.
 */
#ifndef SV_DECAY_H
#define SV_DECAY_H

#include "sv_linattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device workspace of sv_decay_linattn and of sv_decay_linattn_backward for these sizes (either dtype); contents need
 * no preparation.  What a call needs does for every call with no more batches, heads and tokens and the same d.  Pure host functions; 0 for
 * unsupported arguments. */
size_t sv_decay_linattn_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d);
size_t sv_decay_linattn_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d);

/* Whole sequences (prompts, training).  S_in: fp32 [B][H][d][d], the state each sequence begins from, or NULL (zeros).  S_out:
 * receives the state behind its last token, or NULL; may be S_in. */
sv_status sv_decay_linattn(const void *Q, const void *K, const void *V, const sv_tensor_desc *qkv,
                           const float *log_decay, const int32_t *lengths, float scale,
                           const float *S_in, float *S_out, void *O, const sv_tensor_desc *o,
                           void *workspace, size_t workspace_bytes, void *stream);

/* One token of each of B sequences (N = 1), states in a pool of n_slots: S_in, S_out are fp32 [n_slots][H][d][d], row b works on
 * slot slots[b] (int32 [B], device; NULL: slot b, then n_slots >= B).  S_out may be S_in (the step is committed in place) or
 * another pool (a step that can be taken back): slots that no row names are left as they are.  A row whose slot is outside
 * [0, n_slots) is idle: nothing of it is read, and its row of O is left as it is.  A slot named twice serves the first row that
 * names it; the later ones are idle. */
sv_status sv_decay_linattn_token(const void *Q, const void *K, const void *V, const sv_tensor_desc *qkv,
                                 const float *log_decay, const int32_t *slots, int32_t n_slots, float scale,
                                 const float *S_in, float *S_out, void *O, const sv_tensor_desc *o, void *stream);

/* Gradients of sv_decay_linattn for Q, K, V and S_in.  dO: gradient of O.  S_in: as given to the forward call (NULL: zeros).
 * dS_out: gradient of S_out, or NULL (zeros).  dQ, dK, dV (described by qkv) are written at the sequences' tokens; dS_in receives
 * the gradient of S_in, or NULL.  dS_in must not be dS_out. */
sv_status sv_decay_linattn_backward(const void *Q, const void *K, const void *V, const sv_tensor_desc *qkv,
                                    const void *dO, const sv_tensor_desc *o,
                                    const float *log_decay, const int32_t *lengths, float scale,
                                    const float *S_in, const float *dS_out,
                                    void *dQ, void *dK, void *dV, float *dS_in,
                                    void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SV_DECAY_H */
