"""Statistics of the group norm where sums are hardest: constant groups, groups far from zero, and numbers whose squares fp32 does not hold; each for groups that a workgroup
holds and for streamed ones, which have to agree with 64 bits alike.

Bounds: sums are of fp64, of at most 2^21 numbers, off by less than 2^11 fp64 roundings (2^-42 of the terms).  So the mean is off by its rounding to fp32, and rstd by its own;
what is left of the sums' errors is 1e-6 of the mean's distance from the numbers and 2 % of a rounding of rstd."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from tests.gpu_util import say
from tests.selective_util import E, U, draw, f64, like, space

pytestmark = pytest.mark.gpu

# rows, d, groups: held by one workgroup in units of 16, 4 and 2 bytes (or 4), and streamed: narrow groups, wide ones whose sums the next launch adds up, wide ones with a
# launch for it, groups across tiles
SHAPES = [(64, 16, 2), (4090, 16, 2), (61, 48, 8), (50, 40, 8), (70000, 16, 2), (1500, 512, 4), (3000, 512, 4), (5000, 520, 1)]
# name, dtype, (level, spread), eps
GROUPS = [
    ("constant", "f32", (10000.123, 0.0), 1e-5), ("constant", "f32", (-65000.7, 0.0), 1e-5), ("constant", "f32", (1234567.9, 0.0), 1e-5), ("constant", "bf16", (1e4, 0.0), 1e-5),
    ("far", "f32", (1e6, 0.1), 1e-5), ("far", "f32", (3e6, 0.25), 1e-5), ("far", "f32", (-1e4, 1e-2), 1e-8), ("far", "bf16", (300.0, 1.0), 1e-5),
    ("large", "f32", (0.0, 3e19), 1e-5), ("large", "bf16", (0.0, 3e19), 1e-5), ("small", "f32", (0.0, 1e-24), 0.0), ("small", "bf16", (0.0, 1e-24), 0.0),
]


def _statistics(x, G, eps):
    """Mean and variance of each group in two passes of 64 bits (numpy adds in pairs), and rstd."""
    B, H, N, d = x.shape
    v = x.reshape(B, H, N, G, -1)
    mean = v.mean((2, 4))
    return mean, (((v - mean[:, :, None, :, None]) ** 2).mean((2, 4)) + float(np.float32(eps))) ** -0.5


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}-{s[2]}")
@pytest.mark.parametrize("kind", GROUPS, ids=lambda k: f"{k[0]}-{k[1]}-{k[2][0]:g}-{k[2][1]:g}")
def test_statistics(kind, shape):
    import torch
    (name, dtype, (level, spread), eps), (N, d, G) = kind, shape
    say(f"group statistics {name} {dtype} {level} {spread} {N}x{d}-{G}")
    B = 2
    x = draw(1, (B, 1, N, d), dtype, scale=spread, shift=level)
    if name != "constant":
        x[1, 0, 0] = level + 40 * spread                              # one sequence begins with rows apart from its others
    y, mean, rstd = like(x), torch.full((B, 1, G), float("nan"), device="cuda"), torch.full((B, 1, G), float("nan"), device="cuda")
    sv.sv_groupnorm(x, sv.desc_of(x), None, None, G, eps, 0, y, sv.desc_of(y), mean, rstd, space(sv.sv_groupnorm_workspace_bytes(B, 1, N, d, G)))
    h = f64(x)
    m, r = _statistics(h, G, eps)
    M, R = (np.repeat(v, d // G, axis=-1)[:, :, None] for v in (m, r))
    off = E * abs(m) + 1e-6 * E / r
    assert (abs(f64(mean) - m) <= off).all(), f"mean off by {np.max(abs(f64(mean) - m) / off):.3g} of the bound"
    assert (abs(f64(rstd) - r) <= 1.02 * E * r).all(), f"rstd off by {np.max(abs(f64(rstd) / r - 1) / E):.3g} roundings"
    # x - mean is rounded once and the mean before it; rstd and the product are
    want = (h - M) * R
    bound = E * (R * (abs(h - M) + 1.01 * abs(M)) + 2.1 * abs(want))
    worst = np.max(abs(f64(y) - want) / (bound + U[dtype] * (abs(want) + bound) + 2.0 ** -125))
    assert worst <= 1, f"y off by {worst:.3g} of the bound"
    if name == "constant":
        assert (f64(mean) == h[:, :, 0, ::d // G]).all() and not f64(y).any()


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}-{s[2]}")
def test_a_group_that_begins_with_an_infinity(shape):
    """Its mean is that infinity, everything else of it NaN, and the other groups are what they were."""
    import torch
    N, d, G = shape
    say(f"group statistics infinity {N}x{d}-{G}")
    x = draw(1, (2, 1, N, d), "f32")
    out = []
    for bad in (False, True):
        if bad:
            x[1, 0, 0, 0] = float("inf")
        y, mean, rstd = like(x), torch.empty((2, 1, G), device="cuda"), torch.empty((2, 1, G), device="cuda")
        sv.sv_groupnorm(x, sv.desc_of(x), None, None, G, 1e-5, 1, y, sv.desc_of(y), mean, rstd, space(sv.sv_groupnorm_workspace_bytes(2, 1, N, d, G)))
        out.append([f64(v) for v in (y, mean, rstd)])
    (y, mean, rstd), (y2, mean2, rstd2) = out
    assert mean2[1, 0, 0] == np.inf and np.isnan(rstd2[1, 0, 0]) and np.isnan(y2[1, 0, :, :d // G]).all()
    y2[1, 0, :, :d // G] = y[1, 0, :, :d // G]
    mean2[1, 0, 0], rstd2[1, 0, 0] = mean[1, 0, 0], rstd[1, 0, 0]
    assert np.array_equal(y, y2) and np.array_equal(mean, mean2) and np.array_equal(rstd, rstd2)
