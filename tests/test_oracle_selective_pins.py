"""Pins of the float64 formulas that the short convolution, the selective scan and the group norm are tested against
(oracle/selective_oracle.py): automatic differentiation of the forward formulas written another way, differences, and cases worked by hand."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import selective_oracle as orc

TOL = dict(rtol=1e-10, atol=1e-11)          # float64: sums of some hundred terms


def _data(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _same(got, want, lengths=None):
    for name, x in want.items():
        y = got[name]
        x = x.detach().numpy()
        if lengths is not None and np.isnan(y).any():
            x = np.where(np.isnan(y), np.nan, x)
        np.testing.assert_allclose(y, x, err_msg=name, **TOL)


@pytest.mark.parametrize("K,act,lengths", [(2, True, None), (3, False, [5, 0, 1]), (4, True, [7, 2, 3])])
def test_convolution(K, act, lengths):
    B, H, N, d = 3, 2, 7, 4
    x, dy, W, b = (_data(i, *s).requires_grad_() for i, s in enumerate([(B, H, N, d), (B, H, N, d), (K, H, d), (H, d)]))
    cache, dcache = _data(5, B, H, K - 1, d).requires_grad_(), _data(6, B, H, K - 1, d)
    n = orc.lengths_of(lengths, B, N)
    y, out = [], []
    for i in range(B):
        ext = torch.cat([cache[i], x[i, :, :n[i]]], dim=1)                                   # [H][K-1+n][d]
        a = F.conv1d(ext.permute(0, 2, 1).reshape(1, H * d, -1), W.permute(1, 2, 0).reshape(H * d, 1, K), b.reshape(-1), groups=H * d) if n[i] else x.new_zeros((1, H * d, 0))
        a = a.reshape(H, d, -1).permute(0, 2, 1)
        y.append(F.pad(F.silu(a) if act else a, (0, 0, 0, N - n[i])))
        out.append(ext[:, n[i]:])
    y, out = torch.stack(y), torch.stack(out)
    grads = torch.autograd.grad((y * dy).sum() + (out * dcache).sum(), [x, cache, W, b])
    a = [v.detach().numpy() for v in (x, dy, W, b, cache, dcache)]
    _same(orc.conv(a[0], a[2], a[3], act, lengths, a[4])[0], {"y": y, "cache_out": out}, lengths)
    _same(orc.conv_backward(*a[:4], act, lengths, a[4], a[5])[0], dict(zip(("dx", "dcache_in", "dW", "db"), grads)), lengths)


def _scan_torch(u, dt, z, Bm, Cm, A, bias, skip, s_in, n):
    """One sequence after the other, whole decays from sums of steps: h_t = exp(A S_t) h_0 + sum_s exp(A (S_t - S_s)) D_s u_s B_s."""
    B, H, N, d = u.shape
    ys, states = [], []
    for b in range(B):
        D = F.softplus(dt[b, :, :n[b]] + bias[:, None])                                      # [H][n][d]
        S = D.cumsum(1)
        rep = H // Bm.shape[1]
        Bb, Cb = Bm[b, :, :n[b]].repeat_interleave(rep, 0), Cm[b, :, :n[b]].repeat_interleave(rep, 0)
        if n[b] == 0:
            ys.append(u.new_zeros((H, N, d)))
            states.append(s_in[b])
            continue
        apart = S[:, :, None] - S[:, None]                                                   # [H][t][s][d]
        t = torch.arange(n[b])
        w = torch.where((t[:, None] >= t[None])[None, :, :, None, None], torch.exp(apart[..., None] * A[:, None, None]), 0.0)
        h = (w * ((D * u[b, :, :n[b]])[..., None] * Bb[:, :, None])[:, None]).sum(2) + torch.exp(S[..., None] * A[:, None]) * s_in[b][:, None]
        y = (h * Cb[:, :, None]).sum(-1) + skip[:, None] * u[b, :, :n[b]]
        if z is not None:
            y = y * F.silu(z[b, :, :n[b]])
        ys.append(F.pad(y, (0, 0, 0, N - n[b])))
        states.append(h[:, -1])
    return torch.stack(ys), torch.stack(states)


@pytest.mark.parametrize("H,G,gate,lengths", [(2, 1, True, None), (4, 2, False, [6, 0, 1]), (3, 3, True, [2, 6, 5])])
def test_scan(H, G, gate, lengths):
    B, N, d, n = 3, 6, 3, 4
    u, dt, dy, z = (_data(i, B, H, N, d).requires_grad_() for i in range(4))
    Bm, Cm = (_data(4 + i, B, G, N, n).requires_grad_() for i in range(2))
    A = (-torch.exp(_data(6, H, d, n))).requires_grad_()
    bias, skip, s_in = (_data(7 + i, *s).requires_grad_() for i, s in enumerate([(H, d), (H, d), (B, H, d, n)]))
    ds_out, held = _data(10, B, H, d, n), orc.lengths_of(lengths, B, N)
    y, s_out = _scan_torch(u, dt, z if gate else None, Bm, Cm, A, bias, skip, s_in, held)
    leaves = {"du": u, "ddt": dt, "dB": Bm, "dC": Cm, "dA": A, "ddt_bias": bias, "dskip": skip, "ds_in": s_in}
    if gate:
        leaves["dz"] = z
    grads = dict(zip(leaves, torch.autograd.grad((y * dy).sum() + (s_out * ds_out).sum(), list(leaves.values()))))
    a = {k: v.detach().numpy() for k, v in dict(u=u, dt=dt, Bm=Bm, Cm=Cm, A=A, dt_bias=bias, skip=skip, s_in=s_in, z=z).items()}
    a["z"] = a["z"] if gate else None
    a["lengths"] = lengths
    _same(orc.scan(**a)[0], {"y": y, "s_out": s_out}, lengths or [N])
    _same(orc.scan_backward(**a, dy=dy.detach().numpy(), ds_out=ds_out.numpy())[0], grads, lengths or [N])


def test_scan_gradients_are_differences():
    rng = np.random.default_rng(3)
    shapes = dict(u=(1, 2, 4, 2), dt=(1, 2, 4, 2), z=(1, 2, 4, 2), Bm=(1, 1, 4, 3), Cm=(1, 1, 4, 3), A=(2, 2, 3), dt_bias=(2, 2), skip=(2, 2), s_in=(1, 2, 2, 3))
    a = {k: rng.standard_normal(s) for k, s in shapes.items()}
    a["A"] = -np.exp(a["A"])
    dy, ds = rng.standard_normal(shapes["u"]), rng.standard_normal(shapes["s_in"])

    def loss():
        r, _ = orc.scan(**a)
        return (r["y"] * dy).sum() + (r["s_out"] * ds).sum()
    g, _ = orc.scan_backward(**a, dy=dy, ds_out=ds)
    names = dict(u="du", dt="ddt", z="dz", Bm="dB", Cm="dC", A="dA", dt_bias="ddt_bias", skip="dskip", s_in="ds_in")
    for k, name in names.items():
        for at in list(np.ndindex(*shapes[k]))[::3]:
            old, step = a[k][at], 1e-5
            a[k][at] = old + step
            up = loss()
            a[k][at] = old - step
            down = loss()
            a[k][at] = old
            assert abs((up - down) / (2 * step) - g[name][at]) < 1e-8 * max(1, abs(g[name][at])), (name, at)


def test_two_tokens_by_hand():
    """dt_bias so that D = log 2 (dt = 0), A = -1: a = 1/2.  h = 8: 4 + log 2 * 3 * 2, then half of it + log 2 * 1 * 5."""
    l = np.log(2)
    one = lambda *v: np.array(v, dtype=np.float64)
    r, _ = orc.scan(u=one(3, 1).reshape(1, 1, 2, 1), dt=np.zeros((1, 1, 2, 1)), z=None, Bm=one(2, 5).reshape(1, 1, 2, 1), Cm=one(1, 10).reshape(1, 1, 2, 1),
                    A=one(-1).reshape(1, 1, 1), dt_bias=None, skip=one(7).reshape(1, 1), s_in=one(8).reshape(1, 1, 1, 1))
    h1 = 4 + 6 * l
    h2 = h1 / 2 + 5 * l
    np.testing.assert_allclose(r["y"].ravel(), [h1 + 21, 10 * h2 + 7], rtol=1e-14)
    np.testing.assert_allclose(r["s_out"].ravel(), [h2], rtol=1e-14)


@pytest.mark.parametrize("groups,act", [(1, True), (3, False), (12, True)])
def test_group_norm(groups, act):
    B, H, N, d = 2, 3, 5, 12
    x, dy = _data(0, B, H, N, d).requires_grad_(), _data(1, B, H, N, d)
    w, b = (_data(2 + i, d).requires_grad_() for i in range(2))
    flat = x.reshape(B * H, N, d).transpose(1, 2)
    a = F.group_norm(flat, groups, w, b, 1e-3).transpose(1, 2).reshape(x.shape)
    y = F.silu(a) if act else a
    grads = torch.autograd.grad((y * dy).sum(), [x, w, b])
    v = [t.detach().numpy() for t in (x, w, b)]
    r, _ = orc.group_norm(*v, groups, 1e-3, act)
    _same(r, {"y": y})
    _same(orc.group_norm_backward(v[0], dy.numpy(), v[1], v[2], groups, r["mean"], r["rstd"], act, 1)[0], dict(zip(("dx", "dw", "db"), grads)))
