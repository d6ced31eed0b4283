"""A run of the selective operators as a model uses them: group norm with its activation over the frames of hidden states, the short convolution
along the tokens, the selective scan, layer norm of its output; whole sequences with their backward pass, and a prompt that goes on
token by token on pools of caches and states.

fp32 throughout.  Each operator is off by at most a few hundred roundings of its terms' magnitudes (the operators' own tests derive them), four
operators and their gradients after one another by 4 * 400 * 2^-24 = 1e-4 of a tensor's largest value; in the 2-norm, where roundings of random sign
add up as their squares, by a tenth of that."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from tests.gpu_util import say
from tests.selective_util import floats, ints, space

pytestmark = pytest.mark.gpu

B, T, HW, D, N16, GROUPS, TAPS = 2, 3, 40, 96, 16, 8, 4
N = T * HW


def _torch():
    import torch
    return torch


def _model():
    torch = _torch()
    m = dict(gw=1 + floats(1, D, scale=0.2), gb=floats(2, D, scale=0.1), W=floats(3, TAPS, 1, D, scale=0.5), cb=floats(4, 1, D, scale=0.1),
             A=-torch.exp(floats(5, 1, D, N16)), bias=floats(6, 1, D) - 2.0, skip=floats(7, 1, D), lw=1 + floats(8, 1, D, scale=0.2), lb=floats(9, 1, D, scale=0.1))
    x = dict(x=floats(10, B, 1, N, D), dt=floats(11, B, 1, N, D), z=floats(12, B, 1, N, D), Bm=floats(13, B, 1, N, N16), Cm=floats(14, B, 1, N, N16))
    return m, x


def _frames(x):
    return x.view(B, T, HW, D)


def _reference(m, x):
    """The same formulas in float64, for automatic differentiation."""
    torch = _torch()
    F = torch.nn.functional
    a = F.group_norm(x["x"].reshape(B * T, HW, D).transpose(1, 2), GROUPS, m["gw"], m["gb"], 1e-5)
    a = F.silu(a.transpose(1, 2).reshape(B, N, D))
    padded = torch.cat([torch.zeros(B, TAPS - 1, D, dtype=torch.float64), a], dim=1)
    c = F.silu(m["cb"][0] + sum(m["W"][j, 0] * padded[:, j:j + N] for j in range(TAPS)))
    step = F.softplus(x["dt"][:, 0] + m["bias"][0])
    h, ys = torch.zeros(B, D, N16, dtype=torch.float64), []
    for t in range(N):
        h = torch.exp(step[:, t, :, None] * m["A"][0]) * h + (step[:, t] * c[:, t])[..., None] * x["Bm"][:, 0, t, None]
        ys.append((h * x["Cm"][:, 0, t, None]).sum(-1) + m["skip"][0] * c[:, t])
    y = torch.stack(ys, dim=1) * F.silu(x["z"][:, 0])
    return F.layer_norm(y, (D,), m["lw"][0], m["lb"][0], 1e-5)[:, None]


class _Buffers:
    def __init__(self, x):
        torch = _torch()
        e = lambda *s: torch.full(s, float("nan"), device="cuda")
        self.a, self.c, self.y, self.out = (e(B, 1, N, D) for _ in range(4))
        self.gm, self.gr, self.lm, self.lr = e(B, T, GROUPS), e(B, T, GROUPS), e(B, 1, N), e(B, 1, N)
        self.cache, self.state = e(B, 1, TAPS - 1, D), e(B, 1, D, N16)
        self.ws_g = space(max(sv.sv_groupnorm_workspace_bytes(B, T, HW, D, GROUPS), sv.sv_groupnorm_backward_workspace_bytes(B, T, HW, D, GROUPS)))
        self.ws_s = space(max(sv.sv_selective_scan_workspace_bytes(B, 1, N, D, N16), sv.sv_selective_scan_backward_workspace_bytes(B, 1, N, D, 1, N16)))
        self.ws_c = space(sv.sv_causal_conv_backward_workspace_bytes(B, 1, N, D))
        self.ws_l = space(sv.sv_layernorm_backward_workspace_bytes(B, 1, N, D))


def _forward(m, x, s, lengths=None):
    d, f = sv.desc_of(x["x"]), sv.desc_of(_frames(x["x"]))
    sv.sv_groupnorm(x["x"], f, m["gw"], m["gb"], GROUPS, 1e-5, 1, s.a, f, s.gm, s.gr, s.ws_g)
    sv.sv_causal_conv(s.a, d, m["W"], m["cb"], TAPS, 1, lengths, None, s.cache, s.c, d)
    sv.sv_selective_scan(s.c, x["dt"], d, x["z"], d, x["Bm"], x["Cm"], sv.desc_of(x["Bm"]), m["A"], m["bias"], m["skip"], lengths, None, s.state, s.y, d, s.ws_s)
    sv.sv_layernorm(s.y, d, m["lw"], m["lb"], 1, 1e-5, s.out, d, s.lm, s.lr)


def _backward(m, x, s, dout):
    torch = _torch()
    d, f, bc = sv.desc_of(x["x"]), sv.desc_of(_frames(x["x"])), sv.desc_of(x["Bm"])
    g = {k: torch.full_like(v, float("nan")) for k, v in {**m, **x}.items()}
    dy, dc, da = (torch.full_like(x["x"], float("nan")) for _ in range(3))
    sv.sv_layernorm_backward(s.y, d, dout, d, m["lw"], 1, s.lm, s.lr, dy, d, g["lw"], g["lb"], s.ws_l)
    sv.sv_selective_scan_backward(s.c, x["dt"], d, x["z"], d, x["Bm"], x["Cm"], bc, dy, d, m["A"], m["bias"], m["skip"], None, None, None, dc, g["dt"], g["z"], g["Bm"],
                                  g["Cm"], None, g["A"], g["bias"], g["skip"], s.ws_s)
    sv.sv_causal_conv_backward(s.a, d, dc, d, m["W"], m["cb"], TAPS, 1, None, None, None, da, d, None, g["W"], g["cb"], s.ws_c)
    sv.sv_groupnorm_backward(x["x"], f, da, f, m["gw"], m["gb"], GROUPS, 1, s.gm, s.gr, g["x"], f, g["gw"], g["gb"], s.ws_g)
    return g


def _near(name, got, want):
    a, b = got.double().cpu().numpy(), want.detach().numpy()
    assert np.abs(a - b).max() <= 1e-4 * np.abs(b).max(), name
    assert np.linalg.norm(a - b) <= 1e-5 * np.linalg.norm(b), name


def test_training_step():
    say("selective layer, forward and backward")
    torch = _torch()
    m, x = _model()
    s = _Buffers(x)
    _forward(m, x, s)
    dout = floats(20, B, 1, N, D)
    grads = _backward(m, x, s, dout)
    leaves = {k: v.double().cpu().requires_grad_() for k, v in {**m, **x}.items()}
    out = _reference(leaves, leaves)
    _near("out", s.out, out)
    for (k, want) in zip(leaves, torch.autograd.grad((out * dout.double().cpu()).sum(), list(leaves.values()))):
        _near(k, grads[k], want)


def test_prompts_go_on_token_by_token():
    """Prompts of 70 and 101 tokens, then the rest one at a time on pools; layer norm of single rows."""
    say("selective layer, prompt and tokens")
    torch = _torch()
    m, x = _model()
    whole = _Buffers(x)
    _forward(m, x, whole)
    d, one, bc = sv.desc_of(x["x"]), sv.desc_of(x["x"][:, :, :1].contiguous()), sv.desc_of(x["Bm"][:, :, :1].contiguous())
    held = [70, 101]
    s = _Buffers(x)
    _forward(m, x, s, ints(held))
    caches, states = torch.full((5, 1, TAPS - 1, D), float("nan"), device="cuda"), torch.full((5, 1, D, N16), float("nan"), device="cuda")
    slot = [3, 1]
    caches[slot], states[slot] = s.cache, s.state
    out = torch.full_like(s.out, float("nan"))
    for b in range(B):
        out[b, :, :held[b]] = s.out[b, :, :held[b]]
    c1, y1, o1 = (torch.empty((B, 1, 1, D), device="cuda") for _ in range(3))
    for step in range(N - min(held)):
        at = [h + step for h in held]
        live = [t < N for t in at]
        slots = ints([slot[b] if live[b] else -1 for b in range(B)])
        row = lambda v: torch.stack([v[b, :, min(at[b], N - 1)] for b in range(B)])[:, :, None].contiguous()
        sv.sv_causal_conv_token(row(whole.a), one, m["W"], m["cb"], TAPS, 1, slots, 5, caches, caches, c1, one)
        sv.sv_selective_scan_token(c1, row(x["dt"]), one, row(x["z"]), one, row(x["Bm"]), row(x["Cm"]), bc, m["A"], m["bias"], m["skip"], slots, 5, states, states, y1, one)
        sv.sv_layernorm(y1, one, m["lw"], m["lb"], 1, 1e-5, o1, one, None, None)
        for b in range(B):
            if live[b]:
                out[b, :, at[b]] = o1[b, :, 0]
    _near("out", out, whole.out.double().cpu())
    _near("state", states[slot], whole.state.double().cpu())
    assert torch.equal(caches[slot], whole.cache)
    assert torch.isnan(caches[[0, 2, 4]]).all() and torch.isnan(states[[0, 2, 4]]).all()


def test_a_graph_of_the_layer_while_an_eager_one_runs():
    """Two captured graphs with a workspace each, replayed in turn with eager calls between them."""
    say("selective layer, two graphs")
    torch = _torch()
    m, x = _model()
    s, eager = [_Buffers(x), _Buffers(x)], _Buffers(x)
    graphs = []
    for k in s:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            st = torch.cuda.current_stream()
            d, f = sv.desc_of(x["x"]), sv.desc_of(_frames(x["x"]))
            sv.sv_groupnorm(x["x"], f, m["gw"], m["gb"], GROUPS, 1e-5, 1, k.a, f, k.gm, k.gr, k.ws_g, stream=st)
            sv.sv_causal_conv(k.a, d, m["W"], m["cb"], TAPS, 1, None, None, k.cache, k.c, d, stream=st)
            sv.sv_selective_scan(k.c, x["dt"], d, x["z"], d, x["Bm"], x["Cm"], sv.desc_of(x["Bm"]), m["A"], m["bias"], m["skip"], None, None, k.state, k.y, d, k.ws_s, stream=st)
        graphs.append(graph)
    for i in range(3):
        x["x"].copy_(floats(30 + i, B, 1, N, D))
        for g in graphs:
            g.replay()
        _forward(m, x, eager)
        torch.cuda.synchronize()
        for k in s:
            assert torch.equal(k.y, eager.y) and torch.equal(k.state, eager.state)
