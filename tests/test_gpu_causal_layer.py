"""The operators together, as a causal layer uses them: q and k rotated by their tokens' places, decayed linear attention over the sequence, each
head's output brought to scale by a layer norm; its gradients; and the same layer token by token on the states that a prompt left.

fp32 tokens against a chain in 64 bits.  The attention's outputs are off by 3e-6 in the 2-norm (test_gpu_decay.py's arithmetic: the
roundings of some hundred terms are independent), rotation and norm by a few 2^-24 of their terms; the norm divides every row by its own
deviation, and rows whose deviation is a third of the root mean square weigh three times as much: 3 x 3e-6 + 1e-6.  Backwards the same errors
pass through the norm, the attention and the rotation once more: twice that."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
import sv_workloads as wl
from oracle import decay_oracle, layer_oracle
from sv_workloads import metrics
from tests.gpu_util import say, to_host

pytestmark = pytest.mark.gpu

EPS, TOL = 1e-5, 1e-5


def _torch():
    import torch
    return torch


def _space(n):
    return _torch().empty(n, dtype=_torch().uint8, device="cuda").fill_(255)


class _Layer:
    """H heads of d features on a grid of places; q, k, v as views of one projection's output."""

    def __init__(self, B, H, grid, d, seed):
        torch = _torch()
        self.B, self.H, self.grid, self.d, self.N, self.scale = B, H, grid, d, int(np.prod(grid)), d ** -0.5
        gen = torch.Generator().manual_seed(seed)
        self.qkv = torch.randn((B, self.N, 3, H, d), generator=gen).cuda()
        self.w, self.b = (1 + 0.2 * torch.randn((H, d), generator=gen)).cuda(), (0.1 * torch.randn((H, d), generator=gen)).cuda()
        self.g = torch.tensor([-(2.0 ** (-1 - 6 * h / max(1, H - 1))) for h in range(H)], device="cuda")
        self.tables = wl.rope_tables_3d_factored(*grid, d)
        self.rope = sv.Rope3D.from_tensors(*(torch.from_numpy(t).cuda() for t in self.tables))
        self.places = layer_oracle.grid_positions(*grid)

    def views(self, x=None):
        x = self.qkv if x is None else x
        return [x[:, :, i].permute(0, 2, 1, 3) for i in range(3)]

    def heads(self, n=None):
        return _torch().zeros((self.B, self.N if n is None else n, self.H, self.d), device="cuda").permute(0, 2, 1, 3)

    def forward(self, positions=None):
        """-> everything that the backward pass needs."""
        torch = _torch()
        q, k, v = self.views()
        rot = torch.empty_like(self.qkv)
        rq, rk, _ = self.views(rot)
        rot[:, :, 2] = self.qkv[:, :, 2]
        rv = self.views(rot)[2]
        sv.sv_rope3d_rotate(q, k, sv.desc_of(q), self.rope, positions, 0, rq, rk, sv.desc_of(rq))
        o, y = self.heads(), self.heads()
        S = torch.empty((self.B, self.H, self.d, self.d), device="cuda")
        ws = _space(sv.sv_decay_linattn_workspace_bytes(self.B, self.H, self.N, self.d))
        sv.sv_decay_linattn(rq, rk, rv, sv.desc_of(rq), self.g, None, self.scale, None, S, o, sv.desc_of(o), ws)
        mean, rstd = (torch.empty((self.B, self.H, self.N), device="cuda") for _ in range(2))
        sv.sv_layernorm(o, sv.desc_of(o), self.w, self.b, self.H, EPS, y, sv.desc_of(y), mean, rstd)
        return dict(rq=rq, rk=rk, rv=rv, o=o, y=y, S=S, mean=mean, rstd=rstd)

    def backward(self, kept, dy, positions=None):
        torch = _torch()
        do = self.heads()
        dw, db = torch.empty_like(self.w), torch.empty_like(self.b)
        ws = _space(sv.sv_layernorm_backward_workspace_bytes(self.B, self.H, self.N, self.d))
        o = kept["o"]
        sv.sv_layernorm_backward(o, sv.desc_of(o), dy, sv.desc_of(dy), self.w, self.H, kept["mean"], kept["rstd"], do, sv.desc_of(do), dw, db, ws)
        grad = torch.empty_like(self.qkv)
        dq, dk, dv = self.views(grad)
        ws = _space(sv.sv_decay_linattn_backward_workspace_bytes(self.B, self.H, self.N, self.d))
        sv.sv_decay_linattn_backward(kept["rq"], kept["rk"], kept["rv"], sv.desc_of(dq), do, sv.desc_of(do), self.g, None, self.scale, None, None,
                                     dq, dk, dv, None, ws)
        sv.sv_rope3d_rotate(dq, dk, sv.desc_of(dq), self.rope, positions, 1, dq, dk, sv.desc_of(dq))
        return dict(dq=dq, dk=dk, dv=dv, dw=dw, db=db)

    def exact(self, dy):
        q, k, v = (to_host(x).astype(np.float64) for x in self.views())
        g, w, b = to_host(self.g), to_host(self.w), to_host(self.b)
        rq, rk = (layer_oracle.rotate(x, self.tables, self.places) for x in (q, k))
        out, _ = decay_oracle.forward(rq, rk, v, g, self.scale)
        y, mean, rstd = layer_oracle.norm(out["o"], w, b, EPS)
        ng, _ = layer_oracle.norm_backward(out["o"], dy, w, mean, rstd, True)
        ag, _ = decay_oracle.backward(rq, rk, v, ng["dx"], g, self.scale)
        dq, dk = (layer_oracle.rotate(ag[n], self.tables, self.places, inverse=True) for n in ("dq", "dk"))
        return dict(y=y, S=out["s_out"], dq=dq, dk=dk, dv=ag["dv"], dw=ng["dw"], db=ng["db"])


@pytest.mark.parametrize("B,H,grid,d", [(2, 3, (3, 7, 9), 64), (1, 4, (2, 5, 13), 112)])
def test_layer_and_its_gradients(B, H, grid, d):
    torch = _torch()
    say(f"causal layer B={B} H={H} {grid} d={d}")
    layer = _Layer(B, H, grid, d, 5)
    dy = torch.randn((B, layer.N, H, d), generator=torch.Generator().manual_seed(6)).cuda().permute(0, 2, 1, 3)
    kept = layer.forward()
    grads = layer.backward(kept, dy)
    torch.cuda.synchronize()
    ref = layer.exact(to_host(dy))
    assert metrics.rel_l2(to_host(kept["y"]), ref["y"]) <= TOL and metrics.rel_l2(to_host(kept["S"]), ref["S"]) <= TOL
    for n in ("dq", "dk", "dv", "dw", "db"):
        assert metrics.rel_l2(to_host(grads[n]), ref[n]) <= 2 * TOL, n
    # places given per token are the grid's: the same bits
    places = torch.from_numpy(np.broadcast_to(layer.places, (B, layer.N, 3)).astype(np.int32).copy()).cuda()
    again = layer.forward(places)
    back = layer.backward(again, dy, places)
    torch.cuda.synchronize()
    assert torch.equal(again["y"], kept["y"]) and all(torch.equal(back[n], grads[n]) for n in grads)


def test_prompt_then_tokens():
    """A prompt of all but the last tokens into a pool's states, then the last ones one by one, each rotated by its own place: the layer's rows."""
    torch = _torch()
    B, H, grid, d, more = 3, 4, (2, 6, 11), 64, 4
    say("causal layer token by token")
    layer = _Layer(B, H, grid, d, 9)
    whole = layer.forward()
    torch.cuda.synchronize()
    first = layer.N - more
    places = torch.from_numpy(np.broadcast_to(layer.places, (B, layer.N, 3)).astype(np.int32).copy()).cuda()
    rq, rk, rv = (x[:, :, :first] for x in (whole["rq"], whole["rk"], whole["rv"]))
    pool = torch.zeros((5, H, d, d), device="cuda")
    begin = torch.empty((B, H, d, d), device="cuda")
    o = layer.heads(first)
    ws = _space(sv.sv_decay_linattn_workspace_bytes(B, H, first, d))
    sv.sv_decay_linattn(rq, rk, rv, sv.desc_of(rq), layer.g, None, layer.scale, None, begin, o, sv.desc_of(o), ws)
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    pool[slots.long()] = begin
    for t in range(first, layer.N):
        one = layer.qkv[:, t:t + 1].clone()
        q, k, v = (one[:, :, i].permute(0, 2, 1, 3) for i in range(3))
        place = places[:, t:t + 1].contiguous()
        sv.sv_rope3d_rotate(q, k, sv.desc_of(q), layer.rope, place, 0, q, k, sv.desc_of(q))
        o1, y1 = layer.heads(1), layer.heads(1)
        sv.sv_decay_linattn_token(q, k, v, sv.desc_of(q), layer.g, slots, 5, layer.scale, pool, pool, o1, sv.desc_of(o1))
        sv.sv_layernorm(o1, sv.desc_of(o1), layer.w, layer.b, H, EPS, y1, sv.desc_of(y1), None, None)
        torch.cuda.synchronize()
        assert metrics.rel_l2(to_host(y1), to_host(whole["y"][:, :, t:t + 1]).astype(np.float64)) <= 2 * TOL, t
    assert metrics.rel_l2(to_host(pool[slots.long()]), to_host(whole["S"]).astype(np.float64)) <= 2 * TOL
