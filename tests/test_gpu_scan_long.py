"""Selective scans at the lengths of segments and chains of long calls, forwards and backwards against 64 bits, at sizes that the oracle can walk: narrow groups in
many waves.  How each case is cut is pinned in PLANS (tests/test_host_scan_cases.py holds the library's plan to it)."""
import numpy as np
import pytest

from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, like, same_bits, spoil
from tests.test_gpu_scan import _backward, _forward, _Grads, _id, _inputs

pytestmark = pytest.mark.gpu

# B, H, N, d, G, n, gate, dtype, layout, lengths, state; (segments, tokens of a segment) forwards and backwards
PLANS = [
    ((1, 1, 1100, 8, 1, 16, True, "bf16", "bnhd", None, True), (138, 8), (138, 8)),                          # chains in spans of sixteen
    ((1, 1, 2050, 8, 1, 8, False, "f32", "bhnd", None, True), (257, 8), (257, 8)),                           # of thirty-two
    ((1, 2, 4100, 8, 2, 16, True, "f32", "bhnd", [4097], True), (342, 12), (342, 12)),
    ((32, 16, 600, 4, 16, 8, True, "f32", "bnhd", [600, 0, 1, 77, 152, 153, 599, 304] * 4, True), (8, 76), (4, 152)),
    ((32, 16, 1300, 8, 16, 8, False, "bf16", "bnhd", None, False), (10, 132), (4, 328)),                     # twice the waves, forwards
    ((16, 16, 700, 8, 16, 16, True, "bf16", "bhnd", [700 - 43 * b for b in range(16)], True), (16, 44), (8, 88)),
    ((24, 16, 900, 4, 16, 16, False, "f32", "bhnd", [900 - 37 * b for b in range(24)], True), (10, 92), (5, 180)),
    ((130, 16, 40, 4, 16, 8, True, "f32", "bnhd", [40 - b % 41 for b in range(130)], True), (1, 40), (1, 40)),  # not cut
    ((130, 16, 36, 8, 16, 16, False, "bf16", "bhnd", None, False), (1, 36), (1, 36)),
]


@pytest.mark.parametrize("case", PLANS, ids=lambda c: _id(c[0]))
def test_forward(case):
    import torch
    c, (segments, per), _ = case
    B, H, N, d, G, n, gate, dtype, layout, lengths, state = c
    say(f"long scan {_id(c)}")
    x = _inputs(c)
    want, bound = orc.scan(*map(f64, x), lengths, per + segments + 8)
    y, s_out = like(x[0]), torch.full((B, H, d, n), float("nan"), device="cuda")
    _forward(c, x, s_out, y)
    check("y", y, want["y"], bound["y"], dtype)
    check("S_out", s_out, want["s_out"], bound["s_out"], "f32")
    y2 = like(x[0])
    _forward(c, x, None, y2)
    same_bits(y, y2)


@pytest.mark.parametrize("case", PLANS, ids=lambda c: _id(c[0]))
def test_backward(case):
    c, _, (segments, per) = case
    B, H, N, d, G, n, gate, dtype, layout, lengths, state = c
    say(f"long scan backward {_id(c)}")
    x = _inputs(c)
    dy, ds_out = draw(20, (B, H, N, d), dtype, "bnhd"), floats(21, B, H, d, n) if state else None
    spoil(dy, lengths)
    # parameters: a segment's tokens, then the segments of all sequences in order; B and C: a wave's tree of six
    depth = 16 + max(H * d // 64 + 1, per + B * segments)
    u, dt, z, Bm, Cm, A, bias, skip, s_in = map(f64, x)
    want, bound = orc.scan_backward(u, dt, z, Bm, Cm, f64(dy), A, bias, skip, s_in, f64(ds_out), lengths, per + segments + 8, depth)
    g = _Grads(x, B, H, d, n)
    _backward(c, x, dy, ds_out, g.args())
    for name, got in g.all.items():
        if got is not None:
            check(name, got, want[name], bound[name], dtype if name in ("du", "ddt", "dz", "dB", "dC") else "f32")
    assert all(v is None or not np.isnan(f64(v)).all() for v in g.all.values())
