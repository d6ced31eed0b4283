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


def _walk_in_chunks(q, k, v, log_decay, begin, lag, chunk):
    """The walk over [H][n][d] tokens `chunk` at a time: row i of a chunk sees l^(i + lag) times the state in front of the chunk and l^(i - j) k_j
    v_j^T of the chunk's rows j <= i.  -> outputs, magnitudes, and the state
    for the rows behind with its magnitude."""
    H, n, d = q.shape
    g = np.asarray(log_decay, dtype=np.float64)
    S = np.zeros((H, d, d)) if begin is None else np.array(begin, dtype=np.float64)
    M, X = np.abs(S), np.zeros((H, d, d))
    o, mag = np.zeros((H, n, d)), np.zeros((H, n, d))
    for at in range(0, n, chunk):
        a, b, c = (x[:, at:at + chunk] for x in (q, k, v))
        m = a.shape[1]
        i = np.arange(m)
        apart = i[:, None] - i[None, :]
        steps = np.maximum(apart, 0) * g[:, None, None]
        W = np.where(apart >= 0, np.exp(steps), 0.0)
        into = (i + lag) * g[:, None]                                  # [H][m]: of the state in front
        behind = (m - lag - i) * g[:, None]                            # of row i in the state behind
        o[:, at:at + m] = np.exp(into)[..., None] * (a @ S) + (W * (a @ b.transpose(0, 2, 1))) @ c
        aa, ab, ac = np.abs(a), np.abs(b), np.abs(c)
        mag[:, at:at + m] = (np.exp(into)[..., None] * (aa @ (M + X) + np.abs(into)[..., None] * (aa @ M))
                             + (W * (1 + np.abs(steps)) * (aa @ ab.transpose(0, 2, 1))) @ ac)
        whole, weight = (m * g)[:, None, None], np.exp(behind)[..., None]
        X = np.exp(whole) * (X + np.abs(whole) * M) + (ab * weight * np.abs(behind)[..., None]).transpose(0, 2, 1) @ ac
        M = np.exp(whole) * M + (ab * weight).transpose(0, 2, 1) @ ac
        S = np.exp(whole) * S + (b * weight).transpose(0, 2, 1) @ c
    return o, mag, S, M + X


def _in_chunks(B, N, log_decay, lengths, walk):
    """walk(b, n) of every sequence b of n tokens."""
    assert np.isfinite(np.asarray(log_decay)).all()
    return [walk(b, int(n)) for b, n in enumerate(np.full(B, N) if lengths is None else np.clip(np.asarray(lengths), 0, N))]


def _placed(parts, shape):
    out = np.zeros(shape)
    for b, x in enumerate(parts):
        out[b, :, :x.shape[1]] = x
    return out


def forward_in_chunks(q, k, v, log_decay, scale=1.0, s_in=None, lengths=None, chunk=256):
    """`forward` for long sequences: the same sums in another order.  Log decays have to be finite."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))

    def walk(b, n):
        return _walk_in_chunks(scale * q[b, :, :n], k[b, :, :n], v[b, :, :n], log_decay, None if s_in is None else s_in[b], 1, chunk)
    r = _in_chunks(q.shape[0], q.shape[2], log_decay, lengths, walk)
    return ({"o": _placed([x[0] for x in r], q.shape), "s_out": np.stack([x[2] for x in r])},
            {"o": _placed([x[1] for x in r], q.shape), "s_out": np.stack([x[3] for x in r])})


def backward_in_chunks(q, k, v, do, log_decay, scale=1.0, s_in=None, ds_out=None, lengths=None, chunk=256):
    """`backward` for long sequences."""
    q, k, v, do = (np.asarray(x, dtype=np.float64) for x in (q, k, v, do))
    T = (lambda s: None if s is None else np.swapaxes(s, -1, -2))

    def walk(b, n):
        fq, fk, fv, fd = (x[b, :, :n] for x in (q, k, v, scale * do))
        rq, rk, rv, rd = (x[:, ::-1] for x in (fq, fk, fv, fd))
        s, ds = None if s_in is None else s_in[b], None if ds_out is None else ds_out[b]
        dq = _walk_in_chunks(fd, fv, fk, log_decay, T(s), 1, chunk)
        dv = _walk_in_chunks(rk, rq, rd, log_decay, ds, 0, chunk)
        dk = _walk_in_chunks(rv, rd, rq, log_decay, T(ds), 0, chunk)
        return ({"dq": dq[0], "dk": dk[0][:, ::-1], "dv": dv[0][:, ::-1], "ds_in": dv[2]},
                {"dq": dq[1], "dk": dk[1][:, ::-1], "dv": dv[1][:, ::-1], "ds_in": dv[3]})
    r = _in_chunks(q.shape[0], q.shape[2], log_decay, lengths, walk)
    return tuple({n: np.stack([x[side][n] for x in r]) if n == "ds_in" else _placed([x[side][n] for x in r], q.shape) for n in ("dq", "dk", "dv", "ds_in")}
                 for side in (0, 1))
