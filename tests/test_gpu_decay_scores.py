"""What the weighted scores of decayed linear attention lose at bf16, head by head.

A score enters an output as two bf16 pieces, like the state: u^2 of a term, u = 2^-8, beside the output's own rounding u |o|.  So with M the sum
of the magnitudes of an output's terms (oracle/decay_oracle.py) the bound is u |o| + (u^2 + 2 u^2 + (N + 2 d + 64) 2^-24) M for every length, and in the
2-norm nothing but the output's rounding shows, at most u / sqrt 3 = 2.26e-3."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import decay_oracle as orc
from sv_workloads import metrics
from tests.gpu_util import say, to_host
from tests.test_gpu_decay import E, U, _backward, _draw, _host, _prompt, _states, _torch

pytestmark = pytest.mark.gpu


def _check(got, ref, mag, N, d, what):
    got = _host(got)
    tol = U * np.abs(ref) + (3 * U * U + (N + 2 * d + 64) * E) * mag
    bad = ~(np.abs(got - ref) <= tol + 1e-37)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound"
    for h in range(ref.shape[1]):
        assert metrics.rel_l2(got[:, h], ref[:, h]) <= U / np.sqrt(3), (what, h, metrics.rel_l2(got[:, h], ref[:, h]))


@pytest.mark.parametrize("d", [32, 64, 112, 128])
def test_short_memories_are_as_exact_as_long_ones(d):
    """Heads that remember one, three, twenty and a thousand tokens, over several chunks; each by itself."""
    torch = _torch()
    B, H, N, scale = 1, 4, 301, 0.3
    say(f"decay scores d={d}")
    q, k, v, do = _draw(111, B, H, N, d, "bf16", "bnhd", 4)
    g = torch.tensor([-1.0, -0.3, -0.05, -0.001], device="cuda")
    host = [_host(x) for x in (q, k, v)]
    ref, mag = orc.forward(*host, _host(g), scale)
    o, _ = _prompt(q, k, v, g, None, scale, None)
    _check(o, ref["o"], mag["o"], N, d, "o")
    ref, mag = orc.backward(*host, _host(do), _host(g), scale)
    got = _backward(q, k, v, do, g, None, scale, None, None)
    for n in ("dq", "dk", "dv"):
        _check(got[n], ref[n], mag[n], N, d, n)


@pytest.mark.parametrize("d", [32, 64, 112, 128])
def test_padding_does_not_change_a_sequence(d):
    """Ten tokens give the same bits in a row of 10, of 64 and of 200."""
    torch = _torch()
    B, H, n = 3, 2, 10
    say(f"decay padding d={d}")
    q, k, v, do = _draw(112, B, H, 200, d, "bf16", "bhnd", 4)
    g, s_in, ds = torch.tensor([-0.5, -0.01], device="cuda"), _states(15, B, H, d, d), _states(16, B, H, d, d)
    seen = []
    for N in (n, 64, 200):
        cut = [x[:, :, :N] for x in (q, k, v, do)]
        o, s = _prompt(*cut[:3], g, [n] * B, 0.3, s_in)
        grads = _backward(*cut, g, [n] * B, 0.3, s_in, ds)
        seen.append([to_host(x[:, :, :n]) for x in (o, grads["dq"], grads["dk"], grads["dv"])] + [to_host(s), to_host(grads["ds_in"])])
    for other in seen[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(seen[0], other))
