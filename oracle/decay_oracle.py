"""Float64 oracle of decayed causal linear attention (test infrastructure): the recurrences of include/sv_decay.h, token by token,

    S_t = l S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   l = exp(log_decay[h])

with their gradients, and beside every result the sums of the magnitudes of its terms, from which the tests derive how far a result in
fewer bits may be off.  A term that passes through n decays carries n |log_decay| more of a relative error (the exponent's), so the
magnitudes count each term (1 + n |log_decay|) times."""
from __future__ import annotations

import numpy as np


def _decays(log_decay):
    with np.errstate(invalid="ignore"):
        g = np.asarray(log_decay, dtype=np.float64)
    l = np.exp(g)
    return l[None, :, None, None], np.where(np.isinf(g), 0.0, np.abs(g))[None, :, None, None]


class _Carry:
    """A state, the magnitude of its terms and their exponents' share of it."""

    def __init__(self, begin, shape, log_decay):
        self.l, self.g = _decays(log_decay)
        self.s = np.zeros(shape) if begin is None else np.array(begin, dtype=np.float64)
        self.m = np.abs(self.s)
        self.w = np.zeros(shape)

    def decay(self, live):
        l = np.where(live, self.l, 1.0)
        self.w = np.where(live, l * (self.w + self.g * self.m), self.w)
        self.s, self.m = l * self.s, l * self.m

    def add(self, a, b, live):
        x = np.where(live, a[..., :, None] * b[..., None, :], 0.0)
        self.s, self.m = self.s + x, self.m + np.abs(x)

    @property
    def size(self):
        return self.m + self.w


def _tokens(x, keep):
    return np.where(keep[:, None, :, None], np.asarray(x, dtype=np.float64), 0.0)


def _keep(lengths, B, N):
    n = np.full(B, N) if lengths is None else np.clip(np.asarray(lengths), 0, N)
    return np.arange(N)[None, :] < n[:, None]


def forward(q, k, v, log_decay, scale=1.0, s_in=None, lengths=None):
    """-> o, s_out and their magnitudes; rows behind a sequence's length are zeros."""
    B, H, N, d = q.shape
    keep = _keep(lengths, B, N)
    q, k, v = (_tokens(x, keep) for x in (q, k, v))
    S = _Carry(s_in, (B, H, d, d), log_decay)
    o, mag = np.zeros((B, H, N, d)), np.zeros((B, H, N, d))
    for t in range(N):
        live = keep[:, t][:, None, None, None]
        S.decay(live)
        S.add(k[:, :, t], v[:, :, t], live)
        o[:, :, t] = scale * np.einsum("bhk,bhkv->bhv", q[:, :, t], S.s)
        mag[:, :, t] = abs(scale) * np.einsum("bhk,bhkv->bhv", np.abs(q[:, :, t]), S.size)
    return {"o": o, "s_out": S.s}, {"o": mag, "s_out": S.size}


def backward(q, k, v, do, log_decay, scale=1.0, s_in=None, ds_out=None, lengths=None):
    """-> dq, dk, dv, ds_in and their magnitudes."""
    B, H, N, d = q.shape
    keep = _keep(lengths, B, N)
    q, k, v, do = (_tokens(x, keep) for x in (q, k, v, do))
    do = scale * do
    out = {n: np.zeros((B, H, N, d)) for n in ("dq", "dk", "dv")}
    mag = {n: np.zeros((B, H, N, d)) for n in ("dq", "dk", "dv")}
    S = _Carry(s_in, (B, H, d, d), log_decay)
    for t in range(N):
        live = keep[:, t][:, None, None, None]
        S.decay(live)
        S.add(k[:, :, t], v[:, :, t], live)
        out["dq"][:, :, t] = np.einsum("bhkv,bhv->bhk", S.s, do[:, :, t])
        mag["dq"][:, :, t] = np.einsum("bhkv,bhv->bhk", S.size, np.abs(do[:, :, t]))
    G = _Carry(ds_out, (B, H, d, d), log_decay)
    for t in range(N - 1, -1, -1):
        live = keep[:, t][:, None, None, None]
        G.add(q[:, :, t], do[:, :, t], live)
        out["dk"][:, :, t] = np.einsum("bhkv,bhv->bhk", G.s, v[:, :, t])
        out["dv"][:, :, t] = np.einsum("bhkv,bhk->bhv", G.s, k[:, :, t])
        mag["dk"][:, :, t] = np.einsum("bhkv,bhv->bhk", G.size, np.abs(v[:, :, t]))
        mag["dv"][:, :, t] = np.einsum("bhkv,bhk->bhv", G.size, np.abs(k[:, :, t]))
        G.decay(live)
    out["ds_in"], mag["ds_in"] = G.s, G.size
    return out, mag
