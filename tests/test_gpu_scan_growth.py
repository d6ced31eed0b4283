"""Selective scans over several segments in which a segment multiplies a state by more than fp32 holds (A > 0), or by less (far decays of large
states), against 64 bits.  The results are ordinary numbers: what is multiplied is as small, or as large, to begin from.

The bounds are those of oracle/selective_oracle.py.  A segment's sum of steps is one of at most `per` additions, and the sums of at most `segments`
segments follow one another: that is the spread."""
import numpy as np
import pytest

from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, like
from tests.test_gpu_scan import _backward, _forward, _Grads

pytestmark = pytest.mark.gpu

QUIET = -13.8                                                         # softplus of it is 1e-6

# B, H, N, d, G, n, gate, dtype, layout, lengths, state; then the burst's tokens and step, and tokens of a segment and segments (the larger of both directions)
CASES = [
    ((1, 1, 300, 64, 1, 16, True, "bf16", "bhnd", None, True), (40, 48), 12.0, 8, 38),
    ((1, 1, 300, 64, 1, 16, False, "f32", "bhnd", None, True), (40, 48), 12.0, 8, 38),
    ((2, 2, 300, 36, 2, 8, False, "f32", "bnhd", [300, 211], True), (44, 53), 12.0, 8, 38),
    ((2, 1, 1100, 8, 1, 8, True, "bf16", "bnhd", None, True), (803, 812), 12.0, 8, 138),
    ((32, 16, 1300, 4, 16, 8, True, "f32", "bnhd", None, True), (2, 130), 0.54, 328, 10),
    ((32, 16, 700, 8, 16, 8, False, "bf16", "bnhd", None, True), (2, 90), 1.25, 176, 8),
    ((130, 16, 140, 4, 16, 8, True, "f32", "bnhd", None, True), (2, 130), 0.54, 140, 1),
]


def _id(c):
    B, H, N, d, G, n, gate, dtype = c[0][:8]
    return f"{B}x{H}x{N}x{d}-n{n}{'-gate' if gate else ''}-{dtype}"


def _inputs(case, seed, rate, begin, loud):
    """One half of the states at `rate`, the other at decays; steps of 1e-6 outside of the burst.  `loud`: the tokens behind the burst
    add to the states."""
    import torch
    (B, H, N, d, G, n, gate, dtype, layout, lengths, _), (t0, t1), step = case[:3]
    u, dt = draw(seed, (B, H, N, d), dtype, layout), draw(seed + 1, (B, H, N, d), dtype, layout, scale=0.01, shift=QUIET)
    dt[:, :, t0:t1] += step - QUIET
    u[:, :, :t1] = 0
    if not loud:
        u[:] = 0
    z = draw(seed + 2, (B, H, N, d), dtype, "bhnd") if gate else None
    Bm, Cm = draw(seed + 3, (B, G, N, n), dtype, layout), draw(seed + 4, (B, G, N, n), dtype, layout)
    A = -torch.exp(floats(seed + 5, H, d, n, scale=0.3))
    A[:, :, ::2] = rate
    S = begin * floats(seed + 6, B, H, d, n)
    return u, dt, z, Bm, Cm, A, None, floats(seed + 7, H, d), S


def _compare(case, x, dy, ds_out):
    import torch
    c, _, _, per, segments = case
    B, H, N, d, G, n, gate, dtype, _, lengths, _ = c
    spread = per + segments + 8
    want, bound = orc.scan(*map(f64, x), lengths, spread)
    y, s_out = like(x[0]), torch.full((B, H, d, n), float("nan"), device="cuda")
    _forward(c, x, s_out, y)
    check("S_out", s_out, want["s_out"], bound["s_out"], "f32")
    check("y", y, want["y"], bound["y"], dtype)
    u, dt, z, Bm, Cm, A, bias, skip, s_in = map(f64, x)
    depth = 16 + max(H * d // 64 + 1, per + B * segments)
    want, bound = orc.scan_backward(u, dt, z, Bm, Cm, f64(dy), A, bias, skip, s_in, f64(ds_out), lengths, spread, depth)
    g = _Grads(x, B, H, d, n)
    _backward(c, x, dy, ds_out, g.args())
    for name, got in g.all.items():
        if got is not None:
            check(name, got, want[name], bound[name], dtype if name in ("du", "ddt", "dz", "dB", "dC") else "f32")


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_states_that_grow(case):
    """States of 1e-30 that a burst of tokens makes 1e11 to 1e25, and gradients of 1e-30 behind it that it makes as large in front."""
    say(f"scan growth {_id(case)}")
    c, (t0, t1) = case[0], case[1]
    B, H, N, d, G, n, gate, dtype = c[:8]
    x = _inputs(case, 1, 1.0, 1e-30, True)
    dy = draw(20, (B, H, N, d), dtype, "bnhd")
    dy[:, :, t0:] *= 1e-30
    _compare(case, x, dy, 1e-30 * floats(21, B, H, d, n))


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_large_states_that_decay_far(case):
    """States of 1e30 that a burst makes 1e-9 to 1e-26, with nothing added to them, and gradients of 1e24 that it makes 1e-15 to 1e-32: they are these numbers."""
    say(f"scan far decays {_id(case)}")
    B, H, N, d, G, n, gate, dtype = case[0][:8]
    x = _inputs(case, 2, -1.0, 1e30, False)
    x[5][:, :, 1::2] = -0.95
    _compare(case, x, draw(20, (B, H, N, d), dtype, "bnhd", scale=0.0), 1e24 * floats(21, B, H, d, n))


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("n", [8, 16])
def test_a_state_of_nothing_stays_one(n, gate):
    """Bursts past any number fp32 has, on states and gradients that are zero."""
    import torch
    say(f"scan growth of nothing n{n}")
    case = ((1, 1, 300, 64, 1, n, gate, "f32", "bhnd", None, True), (40, 80), 80.0, 8, 38)
    u, dt, z, Bm, Cm, A, _, skip, S = _inputs(case, 3, 1.0, 0.0, True)
    dy = draw(20, (1, 1, 300, 64), "f32")
    dy[:, :, 40:] = 0
    x = (u, dt, z, Bm, Cm, A, None, skip, S)
    y, s_out, g = like(u), torch.empty_like(S), _Grads(x, 1, 1, 64, n)
    _forward(case[0], x, s_out, y)
    _backward(case[0], x, dy, None, g.args())
    assert not f64(y)[:, :, :80].any() and np.isfinite(f64(y)).all() and np.isfinite(f64(s_out)).all() and f64(s_out).any()
    for name, got in g.all.items():
        if got is not None:
            assert np.isfinite(f64(got)).all(), name
    assert not f64(g.all["ddt"]).any() and f64(g.all["du"])[:, :, :40].any()
