"""Pins of the float64 recurrences that decayed attention, rotation and layer norm are tested against (oracle/decay_oracle.py,
oracle/layer_oracle.py): the same results from whole score matrices, from automatic differentiation, and worked by hand."""
import numpy as np
import pytest
import torch

from oracle import decay_oracle, layer_oracle

TOL = dict(rtol=1e-11, atol=1e-11)          # float64: sums of some hundred terms


def _data(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _scores_form(q, k, v, g, scale, s_in, lengths):
    """o and s_out from the whole matrix of decayed scores, no state in between."""
    B, H, N, d = q.shape
    o, s_out = torch.zeros_like(q), []
    for b in range(B):
        n = N if lengths is None else max(0, min(N, lengths[b]))
        row, states = [], []
        for h in range(H):
            t = torch.arange(n, dtype=torch.float64)
            apart = t[:, None] - t[None, :]
            decay = torch.where(apart >= 0, torch.exp(torch.clamp(apart, min=0) * g[h]), 0.0)
            out = ((q[b, h, :n] @ k[b, h, :n].T) * decay) @ v[b, h, :n]
            old = torch.zeros(d, d, dtype=torch.float64) if s_in is None else s_in[b, h]
            out = out + torch.exp((t + 1) * g[h])[:, None] * (q[b, h, :n] @ old)
            row.append(torch.cat([scale * out, torch.zeros(N - n, d, dtype=torch.float64)]))
            states.append(torch.exp(n * g[h]) * old + (k[b, h, :n] * torch.exp((n - 1 - t) * g[h])[:, None]).T @ v[b, h, :n])
        o[b] = torch.stack(row)
        s_out.append(torch.stack(states))
    return o, torch.stack(s_out)


@pytest.mark.parametrize("B,H,N,d,state,lengths", [(1, 2, 1, 4, True, None), (2, 3, 37, 8, True, None), (3, 2, 20, 8, False, [20, 0, 7])])
def test_recurrence_is_the_decayed_score_matrix(B, H, N, d, state, lengths):
    q, k, v, do = (_data(i, B, H, N, d).requires_grad_() for i in range(4))
    s_in = _data(5, B, H, d, d).requires_grad_() if state else None
    ds_out = _data(6, B, H, d, d)
    g = -torch.linspace(0.0, 0.7, H, dtype=torch.float64)
    o, s_out = _scores_form(q, k, v, g, 0.3, s_in, lengths)
    n = np.full(B, N) if lengths is None else np.asarray(lengths)
    kept = torch.tensor(np.arange(N)[None, :] < n[:, None])[:, None, :, None]
    loss = (o * torch.where(kept, do, 0.0)).sum() + (s_out * ds_out).sum()
    leaves = [q, k, v] + ([s_in] if state else [])
    grads = dict(zip(("dq", "dk", "dv", "ds_in"), torch.autograd.grad(loss, leaves)))
    arrays = [x.detach().numpy() for x in (q, k, v, do)]
    begin = s_in.detach().numpy() if state else None
    ref, _ = decay_oracle.forward(*arrays[:3], g.numpy(), 0.3, begin, lengths)
    np.testing.assert_allclose(ref["o"], o.detach().numpy(), **TOL)
    np.testing.assert_allclose(ref["s_out"], s_out.detach().numpy(), **TOL)
    back, _ = decay_oracle.backward(*arrays, g.numpy(), 0.3, begin, ds_out.numpy(), lengths)
    for name, x in grads.items():
        np.testing.assert_allclose(back[name], x.numpy(), err_msg=name, **TOL)


def test_two_tokens_by_hand():
    """l = 1/2, d = 1: S = 8 before; k v = 2 * 3, then 1 * 5: S = 4 + 6 = 10, then 5 + 5 = 10; o = 2 S q with q = 1, then 3."""
    one = lambda *x: np.array(x, dtype=np.float64).reshape(1, 1, -1, 1)
    ref, _ = decay_oracle.forward(one(1, 3), one(2, 1), one(3, 5), np.log([0.5]), 2.0, np.full((1, 1, 1, 1), 8.0))
    np.testing.assert_allclose(ref["o"].ravel(), [20.0, 60.0], **TOL)
    np.testing.assert_allclose(ref["s_out"].ravel(), [10.0], **TOL)
    back, _ = decay_oracle.backward(one(1, 3), one(2, 1), one(3, 5), one(1, 1), np.log([0.5]), 2.0, np.full((1, 1, 1, 1), 8.0))
    # G of the second state: 2 * 3 = 6; of the first: 2 * 1 + 6 / 2 = 5; dq = 2 S, dk = G v, dv = G k, dS = 5 / 2
    for name, x in (("dq", [20, 20]), ("dk", [15, 30]), ("dv", [10, 6]), ("ds_in", [2.5])):
        np.testing.assert_allclose(back[name].ravel(), x, err_msg=name, **TOL)


def test_no_memory_and_whole_memory():
    q, k, v = (_data(i, 1, 2, 9, 4).numpy() for i in range(3))
    ref, _ = decay_oracle.forward(q, k, v, np.array([-np.inf, 0.0]))
    own = (q * k).sum(-1, keepdims=True) * v
    np.testing.assert_allclose(ref["o"][:, 0], own[:, 0], **TOL)                     # the token itself alone
    np.testing.assert_allclose(ref["s_out"][0, 0], np.outer(k[0, 0, -1], v[0, 0, -1]), **TOL)
    np.testing.assert_allclose(ref["s_out"][0, 1], k[0, 1].T @ v[0, 1], **TOL)       # plain linear attention


def test_rotation_is_a_complex_product_and_its_inverse():
    frames, rows, cols, d = 2, 3, 4, 12
    angles = [_data(i, n, p).numpy() for i, (n, p) in enumerate(((frames, 2), (rows, 3), (cols, 1)))]
    tables = [np.stack([np.cos(a), np.sin(a)], -1) for a in angles]
    x = _data(9, 1, 2, frames * rows * cols, d).numpy()
    pos = layer_oracle.grid_positions(frames, rows, cols)
    assert pos[0, 0].tolist() == [0, 0, 0] and pos[0, 1].tolist() == [0, 0, 1] and pos[0, cols].tolist() == [0, 1, 0]
    y = layer_oracle.rotate(x, tables, pos)
    turn = np.concatenate([a[pos[0, :, i]] for i, a in enumerate(angles)], -1)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * turn)
    np.testing.assert_allclose(y[..., 0::2] + 1j * y[..., 1::2], z, **TOL)
    np.testing.assert_allclose(layer_oracle.rotate(y, tables, pos, inverse=True), x, **TOL)
    pos = np.array([[[0, 0, 0], [2, 0, 0], [1, -1, 0]]])                             # two places that are not there
    kept = np.full((1, 2, 3, d), 7.0)
    y = layer_oracle.rotate(x[:, :, :3], tables, pos, kept=kept)
    assert (y[:, :, 1:] == 7.0).all() and not (y[:, :, 0] == 7.0).any()


@pytest.mark.parametrize("per_head", [False, True])
def test_layer_norm_and_its_gradients(per_head):
    B, H, N, d = 2, 3, 5, 8
    x, dy = _data(1, B, H, N, d).requires_grad_(), _data(2, B, H, N, d)
    w, b = (_data(i, H if per_head else 1, d).requires_grad_() for i in (3, 4))
    y = torch.nn.functional.layer_norm(x, (d,), eps=1e-3) * w[None, :, None, :] + b[None, :, None, :]
    dx, dw, db = torch.autograd.grad((y * dy).sum(), (x, w, b))
    a = [t.detach().numpy() for t in (x, w, b)]
    got, mean, rstd = layer_oracle.norm(*a, 1e-3)
    np.testing.assert_allclose(got, y.detach().numpy(), **TOL)
    grads, _ = layer_oracle.norm_backward(a[0], dy.numpy(), a[1], mean, rstd, per_head)
    for name, ref in (("dx", dx), ("dw", dw), ("db", db)):
        np.testing.assert_allclose(grads[name], ref.numpy(), err_msg=name, **TOL)
