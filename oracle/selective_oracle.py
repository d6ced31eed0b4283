"""Float64 oracle of the short causal convolution, the selective scan and the group norm (test infrastructure): the formulas of
include/sv_conv.h, include/sv_scan.h and include/sv_norm.h, with their gradients, and beside every result a bound of what fp32 arithmetic may
be off by, in units of e = 2^-24, from which the tests make their tolerances.

The bounds go term by term.  One rounding costs e of a result, exp and a reciprocal one unit in the last place (2 e); the exponent's product
and constant cost 2 e |x| of exp(x).  So sigmoid(x) is off by (2 |x| + 8) e of itself, silu(x) by that and its factor's error times at most
1.1, silu'(x) = s (1 + x (1 - s)) by (2 |x| + 12) e s (1 + |x| (1 - s)) + 8 |x| s e, and by at most half of x's error.  A sum of n terms
one after the other is off by n e of the terms' magnitudes."""
from __future__ import annotations

import numpy as np


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def silu(x):
    return x * sigmoid(x)


def _slope(x, ex):
    """silu'(x), and how far it may be off where x is off by ex."""
    s = sigmoid(x)
    return s * (1 + x * (1 - s)), 0.5 * ex + (2 * abs(x) + 12) * s * (1 + abs(x) * (1 - s)) + 8 * abs(x) * s


def _activated(a, ea, act):
    return (silu(a), 1.1 * ea + (2 * abs(a) + 8) * abs(silu(a))) if act else (a, ea)


def lengths_of(lengths, B, N):
    return [N] * B if lengths is None else [max(0, min(N, int(n))) for n in lengths]


# ---- short causal convolution ----------------------------------------------------------------------------------------------

def _windows(x, K, cache, n, b):
    """Cache and tokens of sequence b one after the other [H][K-1+n][d]."""
    H, d = x.shape[1], x.shape[3]
    before = np.zeros((H, K - 1, d)) if cache is None else cache[b]
    return np.concatenate([before, x[b, :, :n]], axis=1)


def conv(x, W, bias, act, lengths=None, cache=None):
    """x [B][H][N][d], W [K][H][d], bias [H][d] or None, cache [B][H][K-1][d] or None: {y, cache_out}, bounds.  Rows that are no tokens are NaN."""
    (B, H, N, d), K = x.shape, W.shape[0]
    b = np.zeros((H, d)) if bias is None else bias
    y, e = np.full(x.shape, np.nan), np.full(x.shape, np.nan)
    out = np.zeros((B, H, K - 1, d))
    for i, n in enumerate(lengths_of(lengths, B, N)):
        ext = _windows(x, K, cache, n, i)
        a = b[:, None] + sum(W[j][:, None] * ext[:, j:j + n] for j in range(K))
        m = abs(b[:, None]) + sum(abs(W[j][:, None] * ext[:, j:j + n]) for j in range(K))
        y[i, :, :n], e[i, :, :n] = _activated(a, (K + 1) * m, act)
        out[i] = ext[:, n:]
    return {"y": y, "cache_out": out}, {"y": e, "cache_out": np.zeros_like(out)}


def conv_backward(x, dy, W, bias, act, lengths=None, cache=None, dcache=None, depth=160):
    """Gradients {dx, dcache_in, dW, db}, bounds; `depth`: longest chain of additions of a parameter's gradient."""
    (B, H, N, d), K = x.shape, W.shape[0]
    b = np.zeros((H, d)) if bias is None else bias
    dx, ex = np.full(x.shape, np.nan), np.full(x.shape, np.nan)
    dc, ec = np.zeros((B, H, K - 1, d)), np.zeros((B, H, K - 1, d))
    dW, eW, db, eb = np.zeros(W.shape), np.zeros(W.shape), np.zeros((H, d)), np.zeros((H, d))
    for i, n in enumerate(lengths_of(lengths, B, N)):
        ext = _windows(x, K, cache, n, i)
        da, eda = dy[i, :, :n].copy(), np.zeros((H, n, d))
        if act:
            a = b[:, None] + sum(W[j][:, None] * ext[:, j:j + n] for j in range(K))
            m = abs(b[:, None]) + sum(abs(W[j][:, None] * ext[:, j:j + n]) for j in range(K))
            s, es = _slope(a, (K + 1) * m)
            da, eda = da * s, abs(da) * es + abs(da * s)
        g, eg = np.zeros(ext.shape), np.zeros(ext.shape)
        if dcache is not None:
            g[:, n:] += dcache[i]
            eg[:, n:] += abs(dcache[i])
        for j in range(K):
            g[:, j:j + n] += W[j][:, None] * da
            eg[:, j:j + n] += abs(W[j][:, None]) * (eda + (K + 1) * abs(da))
            dW[j] += (da * ext[:, j:j + n]).sum(1)
            eW[j] += (abs(ext[:, j:j + n]) * (eda + depth * abs(da))).sum(1)
        db += da.sum(1)
        eb += (eda + depth * abs(da)).sum(1)
        dc[i], ec[i] = g[:, :K - 1], eg[:, :K - 1]
        dx[i, :, :n], ex[i, :, :n] = g[:, K - 1:], eg[:, K - 1:]
    return {"dx": dx, "dcache_in": dc, "dW": dW, "db": db}, {"dx": ex, "dcache_in": ec, "dW": eW, "db": eb}


# ---- selective scan --------------------------------------------------------------------------------------------------------

class _Scan:
    """The walk of one call, sequences side by side: what a token takes from u, dt, B and C, the states, and their bounds.  `spread`: how many
    additions a sum of steps D over a run of tokens may have (its error is in the exponent of what goes through the run)."""

    def __init__(self, u, dt, Bm, Cm, A, dt_bias, skip, s_in, lengths, spread):
        B, H, N, d = u.shape
        n, G = A.shape[-1], Bm.shape[1]
        self.A, self.skip, self.n = A, np.zeros((H, d)) if skip is None else skip, n
        self.live = np.arange(N)[None] < np.array(lengths_of(lengths, B, N))[:, None]
        keep = self.live[:, None, :, None]
        clean = lambda x: np.where(keep, x, 0.0)
        bias = np.zeros((H, d)) if dt_bias is None else dt_bias
        self.u, self.x = clean(u), clean(dt + bias[None, :, None])
        self.ex = clean(abs(dt) + abs(bias[None, :, None]))                          # of dt + bias
        self.Bm, self.Cm = (np.repeat(clean(x), H // G, axis=1) for x in (Bm, Cm))   # [B][H][N][n]
        self.G, self.keep = G, keep
        x = self.x
        self.D = np.where(keep, np.maximum(x, 0) + np.log1p(np.exp(-abs(x))), 0.0)
        self.eD = np.where(keep, self.D * (4 * np.maximum(-x, 0) + 14) + sigmoid(x) * self.ex, 0.0)
        self.h, self.m, self.e = ([None] * (N + 1) for _ in range(3))
        self.h[0] = np.zeros((B, H, d, n)) if s_in is None else np.array(s_in, dtype=np.float64)
        self.m[0], self.e[0] = abs(self.h[0]), np.zeros((B, H, d, n))
        self.spread = spread
        for t in range(N):
            a, ea = self.decay(t)
            b = (self.D[:, :, t] * self.u[:, :, t])[..., None] * self.Bm[:, :, t, None]
            eb = (self.eD[:, :, t] * abs(self.u[:, :, t]))[..., None] * abs(self.Bm[:, :, t, None]) + 4 * abs(b)
            self.h[t + 1] = a * self.h[t] + b
            self.m[t + 1] = a * self.m[t] + abs(b)
            self.e[t + 1] = a * (self.e[t] + (ea + 2) * self.m[t]) + eb
        # sum_i C h + skip u, with its magnitude and bound
        self.y = np.stack([(self.h[t + 1] * self.Cm[:, :, t, None]).sum(-1) for t in range(N)], axis=2) + self.skip[None, :, None] * self.u
        self.my = np.stack([(self.m[t + 1] * abs(self.Cm[:, :, t, None])).sum(-1) for t in range(N)], axis=2) + abs(self.skip[None, :, None] * self.u)
        self.ey = np.stack([(self.e[t + 1] * abs(self.Cm[:, :, t, None])).sum(-1) for t in range(N)], axis=2) + (n + 3) * self.my

    def decay(self, t):
        """exp(D A) of token t, and its bound as a share of itself (1 where there is no token)."""
        D, eD, live = self.D[:, :, t, :, None], self.eD[:, :, t, :, None], self.live[:, t, None, None, None]
        x = D * self.A
        return np.exp(x), np.where(live, abs(self.A) * eD + (4 + self.spread) * abs(x) + 3, 0.0)


def scan(u, dt, z, Bm, Cm, A, dt_bias, skip, s_in=None, lengths=None, spread=64):
    """{y, s_out}, bounds; z, dt_bias, skip, s_in may be None.  Rows that are no tokens are NaN."""
    w = _Scan(u, dt, Bm, Cm, A, dt_bias, skip, s_in, lengths, spread)
    y, e = w.y, w.ey
    if z is not None:
        z = np.where(w.keep, z, 0.0)
        y, e = y * silu(z), e * abs(silu(z)) + w.my * abs(silu(z)) * (2 * abs(z) + 10)
    return {"y": np.where(w.keep, y, np.nan), "s_out": w.h[-1]}, {"y": e, "s_out": w.e[-1]}


def scan_backward(u, dt, z, Bm, Cm, dy, A, dt_bias, skip, s_in=None, ds_out=None, lengths=None, spread=64, depth=256):
    """Gradients {du, ddt, dz, dB, dC, ds_in, dA, ddt_bias, dskip}, bounds; `depth`: longest chain of additions of a sum over tokens or channels."""
    w = _Scan(u, dt, Bm, Cm, A, dt_bias, skip, s_in, lengths, spread)
    B, H, N, d = u.shape
    n, G = w.n, w.G
    dy = np.where(w.keep, dy, 0.0)
    g, e = {}, {}
    if z is not None:
        z = np.where(w.keep, z, 0.0)
        s, es = _slope(z, 0 * z)
        g["dz"], e["dz"] = dy * w.y * s, abs(dy) * (abs(s) * (w.ey + 2 * w.my) + es * w.my)
        v, ev = dy * silu(z), abs(dy * silu(z)) * (2 * abs(z) + 10)
    else:
        v, ev = dy, 0 * dy
    u, D, eD, skip = w.u, w.D, w.eD, w.skip
    du, ddt, edu, eddt = (np.zeros(u.shape) for _ in range(4))
    dB, dC, eB, eC = (np.zeros((B, H, N, n)) for _ in range(4))
    dA, eA = np.zeros(A.shape), np.zeros(A.shape)
    G_ = np.zeros((B, H, d, n)) if ds_out is None else np.array(ds_out, dtype=np.float64)
    mG, eG = abs(G_), np.zeros(G_.shape)
    slope = sigmoid(w.x)
    for t in range(N - 1, -1, -1):
        a, ea = w.decay(t)
        C, Bt, vt, evt = w.Cm[:, :, t, None], w.Bm[:, :, t, None], v[:, :, t, :, None], ev[:, :, t, :, None]
        Dt, eDt, ut = D[:, :, t], eD[:, :, t], u[:, :, t]
        G_, mG, eG = G_ + C * vt, mG + abs(C * vt), eG + abs(C) * evt + 3 * (mG + abs(C * vt))
        dC[:, :, t], eC[:, :, t] = (vt * w.h[t + 1]).sum(2), (evt * w.m[t + 1] + abs(vt) * (w.e[t + 1] + depth * w.m[t + 1])).sum(2)
        x = (Dt * ut)[..., None]
        dB[:, :, t] = (G_ * x).sum(2)
        eB[:, :, t] = ((eG + depth * mG) * abs(x) + mG * (eDt * abs(ut))[..., None]).sum(2)
        q, mq = (G_ * Bt).sum(-1), (mG * abs(Bt)).sum(-1)
        eq = (eG * abs(Bt)).sum(-1) + (n + 2) * mq
        p, mp = G_ * a * w.h[t], mG * a * w.m[t]
        ep = a * (eG * w.m[t] + mG * w.e[t]) + (ea + 3) * mp
        dD = (A * p).sum(-1) + ut * q
        mD = (abs(A) * mp).sum(-1) + abs(ut) * mq
        eD_ = (abs(A) * ep).sum(-1) + abs(ut) * eq + (n + 3) * mD
        du[:, :, t] = Dt * q + skip * v[:, :, t]
        edu[:, :, t] = Dt * eq + eDt * mq + abs(skip) * ev[:, :, t] + 3 * (Dt * mq + abs(skip * v[:, :, t]))
        s, xt = slope[:, :, t], w.x[:, :, t]
        ddt[:, :, t], eddt[:, :, t] = dD * s, s * (eD_ + mD * (3 * abs(xt) + w.ex[:, :, t] + 10))
        dA += (Dt[..., None] * p).sum(0)
        eA += (Dt[..., None] * (ep + depth * mp) + eDt[..., None] * mp).sum(0)
        live = w.live[:, t, None, None, None]
        eG = np.where(live, a * (eG + (ea + 2) * mG), eG)
        G_, mG = a * G_, a * mG
    mark = lambda x: np.where(w.keep, x, np.nan)
    ddt, eddt = np.where(w.keep, ddt, 0.0), np.where(w.keep, eddt, 0.0)
    mdt = abs(ddt)
    g.update(du=mark(du), ddt=mark(ddt), ds_in=G_, dA=dA, ddt_bias=ddt.sum((0, 2)), dskip=(v * u).sum((0, 2)))
    e.update(du=edu, ddt=eddt, ds_in=eG, dA=eA, ddt_bias=(eddt + depth * mdt).sum((0, 2)), dskip=((ev + depth * abs(v)) * abs(u)).sum((0, 2)))
    if z is not None:
        g["dz"] = mark(g["dz"])
    for name, x, ex in (("dB", dB, eB), ("dC", dC, eC)):
        g[name] = mark(x.reshape(B, G, H // G, N, n).sum(2))
        e[name] = ex.reshape(B, G, H // G, N, n).sum(2)
    return g, e


# ---- group norm ------------------------------------------------------------------------------------------------------------

def _by_channel(p, d):
    return np.repeat(p, d // p.shape[-1], axis=-1)[:, :, None]


def group_norm(x, w, b, groups, eps, act):
    """x [B][H][N][d], w, b [d] or None: {y, mean, rstd}, bounds."""
    B, H, N, d = x.shape
    w, b = np.ones(d) if w is None else w, np.zeros(d) if b is None else b
    v = x.reshape(B, H, N, groups, -1)
    mean = v.mean((2, 4))
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd = (((v - mean[:, :, None, :, None]) ** 2).mean((2, 4)) + eps) ** -0.5
        M, R = _by_channel(mean, d), _by_channel(rstd, d)
        xh = (x - M) * R
        a = w * xh + b
    # Sums are of fp64, off by less than 2^11 of its roundings of the numbers' mean magnitude A, which is 1e-5 e A: the mean has its own rounding to fp32 beside
    # that, and so has rstd (its sums are of deviations, whose cancellation costs at most 2 % of e).  x - mean, the product with rstd and a are rounded once.
    A = abs(v).mean((2, 4))
    er = np.full(rstd.shape, 1.02)
    ea = abs(w) * (R * (abs(x - M) + abs(M) + 1e-3 * _by_channel(A, d)) + (_by_channel(er, d) + 2) * abs(xh)) + 3 * abs(b)
    y, ey = _activated(a, ea, act)
    return {"y": y, "mean": mean, "rstd": rstd}, {"y": ey, "mean": abs(mean) + 1e-3 * A, "rstd": er * rstd}


def group_norm_backward(x, dy, w, b, groups, mean, rstd, act, depth):
    """Gradients {dx, dw, db} for given statistics, bounds; `depth`: longest chain of additions of a sum over rows."""
    B, H, N, d = x.shape
    w, b = np.ones(d) if w is None else w, np.zeros(d) if b is None else b
    M, R = _by_channel(mean, d), _by_channel(rstd, d)
    xh = (x - M) * R
    exh = R * abs(x - M) + 2 * abs(xh)
    da, eda = dy, np.zeros(dy.shape)
    if act:
        s, es = _slope(w * xh + b, abs(w) * exh + 2 * (abs(w * xh) + abs(b)))
        da, eda = dy * s, abs(dy) * es + abs(dy * s)
    t, et = w * da, abs(w) * (eda + abs(da))

    def level(v, ev):
        sums = lambda q: _by_channel(q.reshape(B, H, N, groups, -1).mean((2, 4)), d)
        return sums(v), sums(ev + depth * abs(v))
    l, el = level(t, et)
    k, ek = level(t * xh, et * abs(xh) + abs(t) * exh)
    dx = R * (t - l - xh * k)
    ex = R * (et + el + abs(xh) * ek + exh * abs(k) + 5 * (abs(t) + abs(l) + abs(xh * k)))
    return ({"dx": dx, "dw": (da * xh).sum((0, 1, 2)), "db": da.sum((0, 1, 2))},
            {"dx": ex, "dw": (eda * abs(xh) + abs(da) * exh + depth * abs(da * xh)).sum((0, 1, 2)), "db": (eda + depth * abs(da)).sum((0, 1, 2))})
