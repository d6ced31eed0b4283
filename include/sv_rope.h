/*
 * sv_rope.h - C ABI of the three-axis rotation of queries and keys on its own (MI355X, gfx950; part of libsvlinattn.so).
 *
 * The _rope3d calls of sv_linattn.h rotate ReLU features inside the attention kernels.  Attention that takes q and k as they are
 * (sv_decay.h, or any other) gets them rotated by this call first, with the same tables and the same pairing: feature pair
 * p = (2p, 2p+1) is turned by the angle of ONE coordinate of the token, its frame (pairs [0, n_t)), its row (the next n_h) or its column (the rest),
 *
 *     y[2p] = x[2p] cos - x[2p+1] sin,    y[2p+1] = x[2p] sin + x[2p+1] cos.
 *
 * The rotation is orthogonal: the backward pass is the rotation by the negative angles, `inverse`.
 */
#ifndef SV_ROPE_H
#define SV_ROPE_H

#include "sv_linattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rotates Q and, if not NULL, K (both described by x) into YQ and YK (described by y; same B, H, N, d and dtype, strides of their
 * own).  YQ may be Q and YK may be K if x and y have the same strides; otherwise outputs must not overlap inputs or each other.
 *  positions   int32 [B][N][3] (frame, row, column), device, 4-byte aligned: each token's place, any places in any order, several
 *              tokens in one place.  A token with a coordinate outside its table (below 0, or frames, rows, cols and above) is
 *              padding: its rows of YQ and YK are left as they are.
 *              NULL: token t of every sequence sits at frame t / (rows*cols), row (t / cols) % rows, column t % cols; then
 *              frames*rows*cols must equal N.
 *  rope        the tables (sv_rope3d): n_t + n_h + n_w = d/2.
 *  inverse     0: by the angles; otherwise by their negatives (the backward pass: dQ, dK from the gradients of YQ, YK).
 * Arithmetic in fp32, one rounding to the tensors' type.  Conventions and errors as in sv_linattn.h; one plain kernel, which may be
 * captured into a HIP graph from the first call on. */
sv_status sv_rope3d_rotate(const void *Q, const void *K, const sv_tensor_desc *x, const sv_rope3d *rope,
                           const int32_t *positions, int inverse, void *YQ, void *YK, const sv_tensor_desc *y,
                           void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SV_ROPE_H */
