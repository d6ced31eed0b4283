"""Group norm (sv_groupnorm) and its backward pass against 64 bits, within the bounds that oracle/selective_oracle.py derives."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, like, place, replayed, same_bits, space

pytestmark = pytest.mark.gpu

EPS = 1e-5
# B, H, N, d, groups, silu, dtype, layout, parameters, level of the rows
CASES = [
    (1, 1, 1, 8, 1, True, "bf16", "bhnd", True, 0.0), (1, 1, 1, 4, 4, False, "f32", "bhnd", True, 0.0), (2, 3, 5, 24, 3, True, "bf16", "apart", True, 1.0),
    (2, 3, 37, 320, 32, True, "bf16", "bnhd", True, 0.3), (3, 1, 901, 320, 32, False, "f32", "bhnd", True, 0.3), (1, 2, 300, 2240, 32, True, "bf16", "bhnd", True, 0.3),
    (1, 1, 700, 40, 40, True, "f32", "apart", False, 0.3), (1, 1, 2500, 16, 2, False, "bf16", "bhnd", True, 5.0), (2, 21, 33, 128, 1, True, "f32", "bnhd", False, 0.3),
    (1, 1, 20, 8192, 64, True, "bf16", "bhnd", True, 0.3), (1, 1, 9, 8192, 8192, False, "f32", "bhnd", True, 0.3), (1, 1, 333, 64, 4, True, "f32", "bhnd", True, 300.0),
    (1, 3, 1560, 140, 2, True, "f32", "bhnd", True, 0.3), (2, 2, 700, 40, 8, True, "bf16", "bnhd", True, 2.0), (1, 2, 3000, 24, 8, False, "bf16", "apart", True, 0.3),
    (1, 1, 2000, 512, 4, True, "bf16", "bhnd", True, 0.3), (1, 1, 130, 2048, 1, True, "bf16", "bhnd", True, 0.3), (3, 7, 100, 256, 1, False, "f32", "bhnd", True, 0.3),
    # streamed: wide groups whose sums go by group (added up by the next launch's workgroups, or by one of their own), groups across tiles, narrow ones
    (2, 1, 5000, 384, 4, True, "bf16", "bhnd", True, 0.3), (2, 3, 2000, 384, 4, True, "bf16", "bnhd", True, 2.0), (1, 2, 1500, 520, 1, False, "bf16", "apart", False, 0.3),
    (1, 3, 1100, 660, 5, True, "f32", "bhnd", True, 0.3), (3, 1, 2500, 296, 8, True, "bf16", "bhnd", True, 0.3), (1, 1, 7000, 72, 1, True, "f32", "apart", True, 0.3),
    (2, 1, 9000, 320, 32, True, "bf16", "bhnd", True, 0.3),
    (5, 40, 3, 48, 6, True, "bf16", "bnhd", True, 0.3), (2, 700, 2, 32, 8, True, "bf16", "bhnd", True, 0.3), (1, 1, 9000, 264, 11, True, "bf16", "bhnd", True, 0.3),
]


def _id(c):
    return f"{c[0]}x{c[1]}x{c[2]}x{c[3]}-{c[4]}{'-silu' if c[5] else ''}-{c[6]}-{c[7]}{'' if c[8] else '-plain'}"


def _inputs(c, seed=1):
    import torch
    B, H, N, d, G, act, dtype, layout, params, level = c
    x = draw(seed, (B, H, N, d), dtype, layout, shift=level)
    w, b = (1 + floats(seed + 1, d, scale=0.3), floats(seed + 2, d, scale=0.2)) if params else (None, None)
    return x, w, b


def _forward(c, x, w, b, y, mean=None, rstd=None, ws=None, stream=None):
    B, H, N, d, G, act = c[:6]
    ws = space(sv.sv_groupnorm_workspace_bytes(B, H, N, d, G)) if ws is None else ws
    sv.sv_groupnorm(x, sv.desc_of(x), w, b, G, EPS, act, y, sv.desc_of(y), mean, rstd, ws, stream=stream)


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_forward(c):
    import torch
    B, H, N, d, G, act, dtype, layout, params, level = c
    say(f"group norm {_id(c)}")
    x, w, b = _inputs(c)
    want, bound = orc.group_norm(f64(x), f64(w), f64(b), G, EPS, act)
    y = like(x)
    mean, rstd = (torch.full((B, H, G), float("nan"), device="cuda") for _ in range(2))
    _forward(c, x, w, b, y, mean, rstd)
    check("mean", mean, want["mean"], bound["mean"], "f32")
    check("rstd", rstd, want["rstd"], bound["rstd"], "f32")
    check("y", y, want["y"], bound["y"], dtype)
    inside = x.clone() if layout == "bhnd" else place(x.cpu(), layout)
    _forward(c, inside, w, b, inside)                                 # in place, statistics not wanted, twice the same bits
    same_bits(y, inside)


def _backward(c, x, dy, w, b, mean, rstd, dx, dw, db, ws=None, stream=None):
    B, H, N, d, G, act = c[:6]
    ws = space(sv.sv_groupnorm_backward_workspace_bytes(B, H, N, d, G)) if ws is None else ws
    sv.sv_groupnorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, b, G, act, mean, rstd, dx, sv.desc_of(dx), dw, db, ws, stream=stream)


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_backward(c):
    import torch
    B, H, N, d, G, act, dtype, layout, params, level = c
    say(f"group norm backward {_id(c)}")
    x, w, b = _inputs(c)
    dy = draw(9, (B, H, N, d), dtype, "bhnd")
    stats, _ = orc.group_norm(f64(x), f64(w), f64(b), G, EPS, act)
    mean, rstd = (torch.from_numpy(stats[k].astype(np.float32)).cuda() for k in ("mean", "rstd"))
    # a thread adds up at most an eighth of the rows (or 64 of many chunks), at most 64 threads one after the other, then the chunks in sixteen runs
    depth = 4 + N // 8 + 64 + 16 + (N // 32 + 1) * B * H // 16
    want, bound = orc.group_norm_backward(f64(x), f64(dy), f64(w), f64(b), G, f64(mean), f64(rstd), act, depth)
    dx, dw, db = like(x), torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    _backward(c, x, dy, w, b, mean, rstd, dx, dw, db)
    check("dx", dx, want["dx"], bound["dx"], dtype)
    check("dw", dw, want["dw"], bound["dw"], "f32")
    check("db", db, want["db"], bound["db"], "f32")
    inside, only = dy.clone(), torch.full((d,), float("nan"), device="cuda")
    _backward(c, x, inside, w, b, mean, rstd, inside, only, None)     # in place of dy, one of the parameters' gradients
    same_bits(dx, inside)
    same_bits(dw, only)
    alone = like(x)
    _backward(c, x, dy, w, b, mean, rstd, alone, None, None)
    same_bits(dx, alone)


@pytest.mark.parametrize("rows", [64, 70000])                         # held by one workgroup, and streamed
def test_statistics_of_constant_and_of_far_rows(rows):
    """A constant group has rstd = eps^-1/2; a group a thousand of its own spreads away keeps its variance."""
    import torch
    x = torch.full((1, 1, rows, 16), 3.0, device="cuda")
    x[..., 8:] = draw(1, (1, 1, rows, 8), "f32", scale=0.25, shift=256.0)
    c = (1, 1, rows, 16, 2, False)
    y, mean, rstd = like(x), torch.empty((1, 1, 2), device="cuda"), torch.empty((1, 1, 2), device="cuda")
    _forward(c, x, None, None, y, mean, rstd)
    want, _ = orc.group_norm(f64(x), None, None, 2, EPS, False)
    assert (f64(y)[..., :8] == 0).all() and float(mean[0, 0, 0]) == 3.0
    np.testing.assert_allclose(f64(mean), want["mean"], rtol=9 * 2.0 ** -24)
    np.testing.assert_allclose(f64(rstd), want["rstd"], rtol=(8 + 0.5 * (9 * 256 / 0.2) ** 2 * 2.0 ** -24) * 2.0 ** -24)


def test_nonfinite_rows_stay_in_their_group():
    c = (2, 2, 40, 64, 4, True, "bf16", "bhnd", True, 0.3)
    x, w, b = _inputs(c)
    y, y2 = like(x), like(x)
    _forward(c, x, w, b, y)
    x[1, 0, 7, 20] = float("nan")
    _forward(c, x, w, b, y2)
    differ = np.isnan(f64(y2))
    assert differ[1, 0, :, 16:32].all() and differ.sum() == 40 * 16
    assert np.array_equal(f64(y)[~differ], f64(y2)[~differ])


@pytest.mark.parametrize("N", [120, 9000])
def test_captured_and_replayed(N):
    import torch
    c = (2, 3, N, 80, 8, True, "bf16", "bnhd", True, 0.3)
    x, w, b = _inputs(c)
    dy = draw(9, (2, 3, N, 80), "bf16", "bnhd")
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    y, dx, mean, rstd, dw, db = like(x), like(x), nan(2, 3, 8), nan(2, 3, 8), nan(80), nan(80)
    ws, wb = space(sv.sv_groupnorm_workspace_bytes(2, 3, N, 80, 8)), space(sv.sv_groupnorm_backward_workspace_bytes(2, 3, N, 80, 8))

    def call(stream):
        _forward(c, x, w, b, y, mean, rstd, ws, stream)
        _backward(c, x, dy, w, b, mean, rstd, dx, dw, db, wb, stream)

    def change(i):
        x.copy_(draw(30 + i, x.shape, "bf16", shift=i))
        dy.copy_(draw(40 + i, x.shape, "bf16"))
    replayed(call, change, [y, mean, rstd, dx, dw, db])


def test_rows_of_a_long_tensor_past_32_bits():
    """Rows 6 MB apart: the last ones lie past 2^31 elements."""
    import torch
    N, stride = 700, 3 << 20
    store = torch.empty(N * stride, dtype=torch.bfloat16, device="cuda")
    far = lambda at: store.as_strided((1, 1, N, 64), (N * stride, N * stride, stride, 1), at)
    c = (1, 1, N, 64, 4, True, "bf16", "bhnd", True, 0.3)
    near, w, b = _inputs(c)
    x, y, y2 = far(0), far(128), like(near)
    x.copy_(near)
    mean, rstd = torch.empty((1, 1, 4), device="cuda"), torch.empty((1, 1, 4), device="cuda")
    _forward(c, x, w, b, y, mean, rstd)
    _forward(c, near, w, b, y2)
    same_bits(y, y2)
    dy = draw(9, (1, 1, N, 64), "bf16")
    dx, dx2, far_dy = far(256), like(near), far(512)
    far_dy.copy_(dy)
    _backward(c, x, far_dy, w, b, mean, rstd, dx, None, None)
    _backward(c, near, dy, w, b, mean, rstd, dx2, None, None)
    same_bits(dx, dx2)
