"""Float64 oracles (test infrastructure) of the operators beside the attention: the three-axis rotation of include/sv_rope.h and the layer norm
of include/sv_norm.h."""
from __future__ import annotations

import numpy as np


def rotate(x, tables, positions, inverse=False, kept=None):
    """x [B][H][N][d]; tables (cs_t, cs_h, cs_w) [places][pairs][2]; positions [B or 1][N][3].  Rows of tokens with a coordinate outside its
    table come from `kept`."""
    x = np.asarray(x, dtype=np.float64)
    pos = np.asarray(positions)
    has = np.ones(pos.shape[:2], dtype=bool)
    for axis, t in enumerate(tables):
        has &= (pos[..., axis] >= 0) & (pos[..., axis] < t.shape[0])
    parts = [np.asarray(t, dtype=np.float64)[np.where(has, pos[..., axis], 0)] for axis, t in enumerate(tables)]
    cs = np.concatenate(parts, axis=2)[:, None]                       # [B][1][N][pairs][2]
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * (cs[..., 0] + (-1j if inverse else 1j) * cs[..., 1])
    y = np.stack([z.real, z.imag], axis=-1).reshape(x.shape)
    return y if has.all() else np.where(has[:, None, :, None], y, kept)


def grid_positions(frames, rows, cols):
    f, r, c = np.meshgrid(np.arange(frames), np.arange(rows), np.arange(cols), indexing="ij")
    return np.stack([f, r, c], axis=-1).reshape(1, -1, 3)


def _parameters(p, H, d, otherwise):
    p = np.full((1, d), otherwise) if p is None else np.asarray(p, dtype=np.float64)
    return np.broadcast_to(p, (H, d))[None, :, None, :]


def norm(x, weight, bias, eps):
    """x [B][H][N][d], weight and bias [1 or H][d] or None -> y, mean, rstd."""
    x = np.asarray(x, dtype=np.float64)
    _, H, _, d = x.shape
    mean = x.mean(-1)
    rstd = 1 / np.sqrt(((x - mean[..., None]) ** 2).mean(-1) + eps)
    xh = (x - mean[..., None]) * rstd[..., None]
    return xh * _parameters(weight, H, d, 1.0) + _parameters(bias, H, d, 0.0), mean, rstd


def norm_backward(x, dy, weight, mean, rstd, per_head):
    """-> dx, dw, db ([1 or H][d]), and the magnitudes of the terms of each."""
    x, dy = (np.asarray(t, dtype=np.float64) for t in (x, dy))
    _, H, _, d = x.shape
    m, r = (np.asarray(t, dtype=np.float64)[..., None] for t in (mean, rstd))
    xh, t = (x - m) * r, _parameters(weight, H, d, 1.0) * dy
    level, along = t.mean(-1, keepdims=True), (t * xh).mean(-1, keepdims=True)
    # what (x - mean) rstd may be off by itself comes from the sizes of x and mean, not of their difference
    size = (np.abs(x) + np.abs(m)) * r
    mag = r * (np.abs(t) + np.abs(t).mean(-1, keepdims=True) + (np.abs(xh) + size) * np.abs(t * xh).mean(-1, keepdims=True)
               + np.abs(xh) * (np.abs(t) * size).mean(-1, keepdims=True))
    over = (0, 2) if per_head else (0, 1, 2)
    out = {"dx": r * (t - level - xh * along), "dw": (dy * xh).sum(over).reshape(-1, d), "db": dy.sum(over).reshape(-1, d)}
    return out, {"dx": mag, "dw": (np.abs(dy) * (np.abs(xh) + size)).sum(over).reshape(-1, d), "db": np.abs(dy).sum(over).reshape(-1, d)}
