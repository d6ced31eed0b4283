"""The selective scan (sv_selective_scan), its token step and its backward pass against 64 bits, within the bounds that
oracle/selective_oracle.py derives."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, ints, like, replayed, same_bits, space, spoil

pytestmark = pytest.mark.gpu

# B, H, N, d, G, n, gate, dtype, layout, lengths, state
CASES = [
    (1, 1, 1, 8, 1, 16, True, "bf16", "bhnd", None, True), (1, 1, 1, 4, 1, 8, False, "f32", "bhnd", None, False),
    (2, 3, 5, 24, 3, 8, True, "bf16", "apart", None, True), (3, 2, 33, 40, 1, 16, False, "bf16", "bnhd", [33, 0, 1], True),
    (4, 4, 41, 112, 2, 16, True, "bf16", "bnhd", [2, 41, 8, 0], False), (4, 6, 40, 36, 2, 8, True, "f32", "apart", [2, 40, 9, 0], True),
    (1, 1, 97, 200, 1, 16, True, "f32", "apart", None, True), (2, 1, 64, 136, 1, 16, True, "f32", "bhnd", [64, 63], True),
    (1, 2, 300, 64, 2, 16, False, "f32", "bhnd", None, True), (1, 1, 517, 72, 1, 16, True, "bf16", "bnhd", None, True),
    (3, 2, 260, 32, 1, 8, False, "f32", "bnhd", [260, 0, 131], True), (1, 1, 20, 8192, 1, 8, True, "bf16", "bhnd", None, False),
    (2, 5, 150, 16, 5, 16, True, "bf16", "bnhd", [32, 150], False),
]


def _id(c):
    return f"{c[0]}x{c[1]}x{c[2]}x{c[3]}-G{c[4]}-n{c[5]}{'-gate' if c[6] else ''}-{c[7]}-{c[8]}{'-ragged' if c[9] else ''}{'-state' if c[10] else ''}"


def _inputs(c, seed=1):
    """(u, dt, z, Bm, Cm, A, dt_bias, skip, s_in): steps of 0.003 to 3, decays of 0.3 to 0.9999."""
    import torch
    B, H, N, d, G, n, gate, dtype, layout, lengths, state = c
    u, dt = draw(seed, (B, H, N, d), dtype, layout), draw(seed + 1, (B, H, N, d), dtype, layout, scale=1.5, shift=-2.0)
    z = draw(seed + 2, (B, H, N, d), dtype, "bhnd") if gate else None
    Bm, Cm = draw(seed + 3, (B, G, N, n), dtype, layout), draw(seed + 4, (B, G, N, n), dtype, layout)
    A = -torch.exp(floats(seed + 5, H, d, n)) * torch.linspace(0.05, 1.0, n, device="cuda")
    for x in (u, dt, z, Bm, Cm):
        if x is not None:
            spoil(x, lengths)
    return u, dt, z, Bm, Cm, A, floats(seed + 6, H, d, scale=0.5), floats(seed + 7, H, d), floats(seed + 8, B, H, d, n) if state else None


def _spread(N):
    """Additions in a sum of steps: a segment's tokens, and the segments it goes on through."""
    return N + 8


def _forward(c, x, s_out, y, ws=None, stream=None, s_in=0, lengths=0):
    u, dt, z, Bm, Cm, A, bias, skip, begin = x
    B, H, N, d, G, n = c[:6]
    ws = space(sv.sv_selective_scan_workspace_bytes(B, H, N, d, n)) if ws is None else ws
    sv.sv_selective_scan(u, dt, sv.desc_of(u), z, sv.desc_of(z) if z is not None else None, Bm, Cm, sv.desc_of(Bm), A, bias, skip,
                         ints(c[9]) if isinstance(lengths, int) else lengths, begin if isinstance(s_in, int) else s_in, s_out, y, sv.desc_of(y), ws, stream=stream)


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_forward(c):
    import torch
    B, H, N, d, G, n, gate, dtype, layout, lengths, state = c
    say(f"scan {_id(c)}")
    x = _inputs(c)
    want, bound = orc.scan(*map(f64, x), lengths, _spread(N))
    y, s_out = like(x[0]), torch.full((B, H, d, n), float("nan"), device="cuda")
    _forward(c, x, s_out, y)
    check("y", y, want["y"], bound["y"], dtype)
    check("S_out", s_out, want["s_out"], bound["s_out"], "f32")
    y2 = like(x[0])
    held = x[-1].clone() if state else None
    _forward(c, x, held, y2, s_in=held)                               # in place (or no S_out), and twice the same bits
    same_bits(y, y2)
    if state:
        same_bits(s_out, held)


def test_forward_without_bias_and_skip():
    c = (2, 2, 19, 48, 1, 16, True, "bf16", "bnhd", None, False)
    u, dt, z, Bm, Cm, A, _, _, _ = _inputs(c)
    want, bound = orc.scan(*map(f64, (u, dt, z, Bm, Cm, A, None, None, None)))
    y = like(u)
    _forward(c, (u, dt, z, Bm, Cm, A, None, None, None), None, y)
    check("y", y, want["y"], bound["y"], "bf16")


class _Grads:
    NAMES = ("du", "ddt", "dz", "dB", "dC", "ds_in", "dA", "ddt_bias", "dskip")

    def __init__(self, x, B, H, d, n):
        import torch
        u, dt, z, Bm, Cm, A, bias, skip, _ = x
        nan = lambda *s: torch.full(s, float("nan"), device="cuda")
        self.all = dict(du=like(u), ddt=like(dt), dz=like(z) if z is not None else None, dB=like(Bm), dC=like(Cm), ds_in=nan(B, H, d, n), dA=nan(H, d, n),
                        ddt_bias=nan(H, d), dskip=nan(H, d))

    def args(self):
        return [self.all[k] for k in self.NAMES]


def _backward(c, x, dy, ds_out, grads, ws=None, stream=None, lengths=0):
    u, dt, z, Bm, Cm, A, bias, skip, begin = x
    B, H, N, d, G, n = c[:6]
    ws = space(sv.sv_selective_scan_backward_workspace_bytes(B, H, N, d, G, n)) if ws is None else ws
    sv.sv_selective_scan_backward(u, dt, sv.desc_of(u), z, sv.desc_of(z) if z is not None else None, Bm, Cm, sv.desc_of(Bm), dy, sv.desc_of(dy), A, bias, skip,
                                  ints(c[9]) if isinstance(lengths, int) else lengths, begin, ds_out, *grads, ws, stream=stream)


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_backward(c):
    B, H, N, d, G, n, gate, dtype, layout, lengths, state = c
    say(f"scan backward {_id(c)}")
    x = _inputs(c)
    dy, ds_out = draw(20, (B, H, N, d), dtype, "bnhd"), floats(21, B, H, d, n) if state else None
    spoil(dy, lengths)
    # sums over channels: a wave's tree of six, then the waves in order; over tokens: a segment's, then the segments in order
    depth = 16 + max(H * d // 64 + 1, N + 2 * B * 128)
    u, dt, z, Bm, Cm, A, bias, skip, s_in = map(f64, x)
    want, bound = orc.scan_backward(u, dt, z, Bm, Cm, f64(dy), A, bias, skip, s_in, f64(ds_out), lengths, _spread(N), depth)
    g = _Grads(x, B, H, d, n)
    _backward(c, x, dy, ds_out, g.args())
    for name, got in g.all.items():
        if got is not None:
            check(name, got, want[name], bound[name], dtype if name in ("du", "ddt", "dz", "dB", "dC") else "f32")
    few = _Grads(x, B, H, d, n)                                       # no gradient of the state, one of the parameters'
    _backward(c, x, dy, ds_out, [few.all[k] if k not in ("ds_in", "dA", "ddt_bias") else None for k in few.NAMES])
    for k in ("du", "ddt", "dB", "dC", "dskip"):
        same_bits(g.all[k], few.all[k])


def test_backward_of_the_state_in_place():
    c = (2, 1, 70, 64, 1, 16, True, "f32", "bhnd", [70, 0], True)
    x = _inputs(c)
    dy, ds_out = draw(20, (2, 1, 70, 64), "f32"), floats(21, 2, 1, 64, 16)
    spoil(dy, [70, 0])
    g, held = _Grads(x, 2, 1, 64, 16), ds_out.clone()
    _backward(c, x, dy, ds_out, g.args())
    again = _Grads(x, 2, 1, 64, 16)
    again.all["ds_in"] = held
    _backward(c, x, dy, held, again.args())
    for k, v in g.all.items():
        same_bits(v, again.all[k])
    same_bits(held[1], ds_out[1])                                     # no tokens: handed through


@pytest.mark.parametrize("rows,pool,H,d,G,n,gate,dtype,elsewhere", [
    (1, 1, 1, 8, 1, 16, True, "bf16", False), (5, 9, 4, 36, 2, 8, False, "f32", True), (12, 12, 2, 112, 2, 16, True, "bf16", True),
    (6, 8, 1, 2240, 1, 16, True, "bf16", False), (3, 5, 1, 8192, 1, 8, False, "f32", True), (5, 6, 5, 64, 5, 16, True, "f32", False),
    (70, 80, 1, 2240, 1, 16, True, "bf16", True), (130, 140, 2, 1100, 2, 8, False, "f32", False)])
def test_token(rows, pool, H, d, G, n, gate, dtype, elsewhere):
    import torch
    say(f"scan token {rows} of {pool} {H}x{d} G{G} n{n} {dtype}")
    u, dt, z, Bm, Cm, A, bias, skip, _ = _inputs((rows, H, 1, d, G, n, gate, dtype, "apart", None, False))
    before = floats(9, pool, H, d, n)
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(5))[:rows].tolist()
    if rows > 4:
        order[1], order[2], order[4] = -1, pool, order[0]             # idle, idle, a slot named twice
    S = before.clone()
    out = torch.full_like(before, float("nan")) if elsewhere else S
    y = like(u)
    sv.sv_selective_scan_token(u, dt, sv.desc_of(u), z, sv.desc_of(z) if gate else None, Bm, Cm, sv.desc_of(Bm), A, bias, skip, ints(order), pool, S, out, y,
                               sv.desc_of(y))
    served, named = f64(y), set()
    expect, bounds = (np.full((pool, H, d, n), np.nan) if elsewhere else f64(before)), np.zeros((pool, H, d, n))
    for r, slot in enumerate(order):
        if not 0 <= slot < pool or slot in named:
            assert np.isnan(served[r]).all()
            continue
        named.add(slot)
        one = [f64(v[r:r + 1]) if v is not None else None for v in (u, dt, z, Bm, Cm)]
        want, bound = orc.scan(*one, f64(A), f64(bias), f64(skip), f64(before[slot:slot + 1]))
        check("y", y[r:r + 1], want["y"], bound["y"], dtype)
        expect[slot], bounds[slot] = want["s_out"][0], bound["s_out"][0]
    check("S_out", out, expect, bounds, "f32")
    for slot in set(range(pool)) - named:                             # the others are left alone
        if not elsewhere:
            same_bits(out[slot], before[slot])


def test_token_steps_are_a_prompt():
    """Without slots row b works on state b; nine steps are the prompt within its bounds."""
    c = (3, 2, 9, 64, 2, 16, True, "f32", "bnhd", None, True)
    x = _inputs(c)
    u, dt, z, Bm, Cm, A, bias, skip, S = x
    want, bound = orc.scan(*map(f64, x))
    y, S = like(u), S.clone()
    for t in range(9):
        one = [v[:, :, t:t + 1] for v in (u, dt, z, Bm, Cm, y)]
        sv.sv_selective_scan_token(one[0], one[1], sv.desc_of(one[0]), one[2], sv.desc_of(one[2]), one[3], one[4], sv.desc_of(one[3]), A, bias, skip, None, 3, S, S,
                                   one[5], sv.desc_of(one[5]))
    check("y", y, want["y"], bound["y"], "f32")
    check("S", S, want["s_out"], bound["s_out"], "f32")


def test_a_prompt_in_pieces():
    c = (2, 1, 400, 72, 1, 16, True, "f32", "bhnd", None, True)
    x = _inputs(c)
    want, bound = orc.scan(*map(f64, x), None, _spread(400))
    u, dt, z, Bm, Cm, A, bias, skip, S = x
    y, S = like(u), S.clone()
    for t0, t1 in ((0, 1), (1, 3), (3, 330), (330, 400)):
        u1, dt1, z1, B1, C1, y1 = (v[:, :, t0:t1] for v in (u, dt, z, Bm, Cm, y))
        _forward((2, 1, t1 - t0, 72, 1, 16, True, "f32", "bhnd", None, True), (u1, dt1, z1, B1, C1, A, bias, skip, S), S, y1)
    check("y", y, want["y"], bound["y"], "f32")
    check("S", S, want["s_out"], bound["s_out"], "f32")


def test_steps_of_every_size():
    """softplus from 1e-26 to 60, decays from 1 - 1e-7 to 0, states that stay as they are (A = 0) or vanish (A = -inf)."""
    import torch
    c = (1, 1, 130, 64, 1, 16, False, "f32", "bhnd", None, True)
    u, _, _, Bm, Cm, A, _, skip, S = _inputs(c)
    dt = torch.linspace(-60, 60, 64, device="cuda").expand(1, 1, 130, 64).contiguous()
    A = A.clone()
    A[:, :, 0], A[:, :, 1] = 0.0, float("-inf")
    y, s_out = like(u), torch.empty_like(S)
    _forward(c, (u, dt, None, Bm, Cm, A, None, skip, S), s_out, y)
    A[:, :, 1] = -1e30                                                # the oracle's products stay numbers
    want, bound = orc.scan(*map(f64, (u, dt, None, Bm, Cm, A, None, skip, S)), None, _spread(130))
    live = [i for i in range(16) if i != 1]
    check("S_out", s_out[..., live], want["s_out"][..., live], bound["s_out"][..., live], "f32")
    assert np.isfinite(f64(y)).all() and np.isfinite(f64(s_out)).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_nonfinite_tokens_leave_earlier_outputs_alone(value):
    c = (1, 1, 300, 64, 1, 16, True, "bf16", "bhnd", None, True)
    x = _inputs(c)
    y, y2 = like(x[0]), like(x[0])
    _forward(c, x, None, y)
    dy, g = draw(20, (1, 1, 300, 64), "bf16"), _Grads(x, 1, 1, 64, 16)
    _backward(c, x, dy, None, g.args())
    x[0][0, 0, 150, 5] = value
    _forward(c, x, None, y2)
    same_bits(y[:, :, :150], y2[:, :, :150])
    others = [i for i in range(64) if i != 5]
    same_bits(y[..., others], y2[..., others])
    assert not np.isfinite(f64(y2)[0, 0, 150:, 5]).any()
    x = _inputs(c)
    dy[0, 0, 150, 5] = value
    bad = _Grads(x, 1, 1, 64, 16)
    _backward(c, x, dy, None, bad.args())
    for k in ("du", "ddt", "dz"):                                     # gradients of later tokens and of other channels
        same_bits(g.all[k][:, :, 151:], bad.all[k][:, :, 151:])
        same_bits(g.all[k][..., others], bad.all[k][..., others])
    same_bits(g.all["dC"][:, :, 151:], bad.all["dC"][:, :, 151:])


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("behind", [True, False])
def test_a_step_that_is_no_number(gate, behind):
    """Token 150 of one channel: no gradient comes back through it, also none of zero, and the later ones are what they were."""
    c = (1, 1, 300, 64, 1, 16, gate, "f32", "bhnd", None, True)
    x = _inputs(c)
    dy = draw(20, (1, 1, 300, 64), "f32")
    if not behind:
        dy[:, :, 150:] = 0
    good, bad = _Grads(x, 1, 1, 64, 16), _Grads(x, 1, 1, 64, 16)
    _backward(c, x, dy, None, good.args())
    x[1][0, 0, 150, 5] = float("nan")
    _backward(c, x, dy, None, bad.args())
    others = [i for i in range(64) if i != 5]
    for k in ("du", "ddt"):
        assert np.isnan(f64(bad.all[k])[0, 0, :150, 5]).all()
        same_bits(good.all[k][..., others], bad.all[k][..., others])
    same_bits(good.all["du"][:, :, 151:], bad.all["du"][:, :, 151:])
    if gate:
        same_bits(good.all["dz"][:, :, :150], bad.all["dz"][:, :, :150])
    assert np.isnan(f64(bad.all["ds_in"])[0, 0, 5]).all()
    same_bits(good.all["ds_in"][:, :, others], bad.all["ds_in"][:, :, others])


def test_captured_and_replayed():
    import torch
    c = (3, 2, 290, 48, 1, 16, True, "bf16", "bnhd", [290, 17, 0], True)
    x = _inputs(c)
    u, Bm = x[0], x[3]
    dy, ds_out, n = draw(20, (3, 2, 290, 48), "bf16", "bnhd"), floats(21, 3, 2, 48, 16), ints([290, 17, 0])
    y, s_out, g = like(u), torch.empty_like(x[-1]), _Grads(x, 3, 2, 48, 16)
    ws = space(sv.sv_selective_scan_workspace_bytes(3, 2, 290, 48, 16))
    wb = space(sv.sv_selective_scan_backward_workspace_bytes(3, 2, 290, 48, 1, 16))

    def call(stream):
        _forward(c, x, s_out, y, ws, stream, lengths=n)
        _backward(c, x, dy, ds_out, g.args(), wb, stream, lengths=n)

    def change(i):
        for k, v in enumerate((u, x[1], x[2], Bm, x[4], dy)):
            v.copy_(draw(30 + 10 * i + k, v.shape, "bf16"))
        n.copy_(ints([[290, 17, 0], [33, 290, 144], [1, 256, 290]][i]))
    replayed(call, change, [y, s_out] + [v for v in g.all.values()])


def test_rows_of_a_long_tensor_past_32_bits():
    """Tokens 6 MB apart: the last ones lie past 2^31 elements."""
    import torch
    N, stride = 700, 3 << 20
    store = torch.empty(N * stride, dtype=torch.bfloat16, device="cuda")
    far = lambda at, d: store.as_strided((1, 1, N, d), (N * stride, N * stride, stride, 1), at)
    c = (1, 1, N, 64, 1, 16, True, "bf16", "bhnd", None, True)
    near = _inputs(c)
    x = [far(128 * i, near[i].shape[-1]) for i in range(5)] + list(near[5:])
    for i in range(5):
        x[i].copy_(near[i])
    y, y2, dy = far(1024, 64), like(near[0]), draw(20, (1, 1, N, 64), "bf16")
    s1, s2 = (torch.empty_like(near[-1]) for _ in range(2))
    _forward(c, x, s1, y)
    _forward(c, near, s2, y2)
    same_bits(y, y2)
    same_bits(s1, s2)
    y.copy_(dy)
    g1, g2 = _Grads(near, 1, 1, 64, 16), _Grads(near, 1, 1, 64, 16)
    for i, k in enumerate(("du", "ddt", "dz", "dB", "dC")):
        g1.all[k] = far(2048 + 128 * i, g1.all[k].shape[-1])
    _backward(c, x, y, None, g1.args())
    _backward(c, near, dy, None, g2.args())
    for k in g1.all:
        same_bits(g1.all[k], g2.all[k])
