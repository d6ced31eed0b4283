"""Selective scans of more sequences than the kernel between segments could have workgroups for: they are not cut, so it does not run, and the call is served."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, like, same_bits, space

pytestmark = pytest.mark.gpu

N, d, n = 2, 2240, 16


def test_forward():
    import torch
    B = 7500
    assert B * d * n // 64 >= 1 << 22
    say(f"scan of {B} sequences")
    u, dt, z = (draw(i, (B, 1, N, d), "bf16") for i in range(3))
    Bm, Cm, A = draw(4, (B, 1, N, n), "bf16"), draw(5, (B, 1, N, n), "bf16"), -torch.exp(floats(6, 1, d, n))

    def run(at):
        x = [v[at] for v in (u, dt, z, Bm, Cm)]
        y = like(x[0])
        D, C = sv.desc_of(x[0]), sv.desc_of(x[3])
        sv.sv_selective_scan(x[0], x[1], D, x[2], D, x[3], x[4], C, A, None, None, None, None, None, y, D, space(sv.sv_selective_scan_workspace_bytes(len(x[0]), 1, N, d, n)))
        return y
    y = run(slice(None))
    for at in (slice(0, 4000), slice(4000, B)):                       # the same sequences in two calls, which are not cut either
        same_bits(y[at], run(at))
    last = slice(B - 3, B)
    want, bound = orc.scan(*(f64(v[last]) for v in (u, dt, z, Bm, Cm)), f64(A), None, None)
    check("y", y[last], want["y"], bound["y"], "bf16")


def test_backward():
    import torch
    B = 3800
    assert 2 * B * d * n // 64 >= 1 << 22
    say(f"scan backward of {B} sequences")
    u, dt, z, dy = (draw(i, (B, 1, N, d), "bf16") for i in range(4))
    Bm, Cm, A = draw(4, (B, 1, N, n), "bf16"), draw(5, (B, 1, N, n), "bf16"), -torch.exp(floats(6, 1, d, n))

    def run(at):
        x = [v[at] for v in (u, dt, z, Bm, Cm, dy)]
        g = [like(v) for v in x[:5]]
        D, C = sv.desc_of(x[0]), sv.desc_of(x[3])
        sv.sv_selective_scan_backward(x[0], x[1], D, x[2], D, x[3], x[4], C, x[5], D, A, None, None, None, None, None, *g, None, None, None, None,
                                      space(sv.sv_selective_scan_backward_workspace_bytes(len(x[0]), 1, N, d, 1, n)))
        return g
    whole = run(slice(None))
    for at in (slice(0, 1800), slice(1800, B)):
        for a, b in zip(whole, run(at)):
            same_bits(a[at], b)
    last = slice(B - 3, B)
    want, bound = orc.scan_backward(*(f64(v[last]) for v in (u, dt, z, Bm, Cm, dy)), f64(A), None, None)
    for name, got in zip(("du", "ddt", "dz", "dB", "dC"), whole):
        check(name, got[last], want[name], bound[name], "bf16")
    assert not any(np.isnan(f64(v)).any() for v in whole)
