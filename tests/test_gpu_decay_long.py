"""Decayed linear attention over long sequences: many chunks in every segment, many segments, and prompts whose tokens pass the caches by.

The bounds are test_gpu_decay.py's, with the scores in two pieces (u^2 M); in the 2-norm, head by head, bf16 outputs are off by no more than their own
rounding, u / sqrt 3, and what is held in fp32 by 3e-6: a state goes through N / 32 roundings of 2^-24 / sqrt 3 or less each, which are
independent: sqrt(33 000 / 32) x 3.4e-8 = 1.1e-6, and as much again for the products.  Heads that forget nothing are among them.  The oracle
looks at some heads of each call, the other heads only have to be finite.

test_host_decay_cases.py holds the cases to what they are here for."""
import numpy as np
import pytest

from oracle import decay_oracle as orc
from sv_workloads import metrics
from tests.gpu_util import say, to_host
from tests.test_gpu_decay import E, U, _backward, _draw, _like, _prompt, _states, _torch

pytestmark = pytest.mark.gpu

# B, H, N, d, dtype, layout, lengths, state
PROMPTS = [
    (2, 32, 33000, 32, "bf16", "bhnd", [33000, 20011], True),
    (1, 32, 33001, 64, "bf16", "bhnd", None, True),
    (1, 20, 30001, 112, "bf16", "packed", None, False),
    (1, 20, 30001, 112, "bf16", "bhnd", None, True),
    (2, 8, 33001, 128, "bf16", "bnhd", [32700, 33001], True),
    (1, 16, 33001, 64, "f32", "packed", None, True),
    (1, 10, 33001, 112, "f32", "bhnd", None, True),
    (1, 8, 33001, 128, "f32", "bhnd", None, False),
]
BACKWARDS = [
    (2, 32, 9001, 32, "bf16", "bhnd", [9001, 5123], True),
    (1, 40, 5001, 64, "bf16", "bnhd", None, True),
    (2, 12, 9001, 112, "bf16", "packed", [9001, 5003], True),
    (1, 12, 9001, 128, "bf16", "bhnd", None, True),
    (1, 40, 5001, 32, "f32", "bhnd", None, True),
    (2, 20, 3001, 64, "f32", "packed", [3001, 2503], True),
    (1, 20, 7001, 112, "f32", "packed", None, True),
    (1, 20, 7001, 128, "f32", "bnhd", None, False),
]


def _id(c):
    return f"B{c[0]}H{c[1]}N{c[2]}d{c[3]}-{c[4]}-{c[5]}{'-ragged' if c[6] else ''}{'' if c[7] else '-nostate'}"


def _decays(H):
    """Memories of one token to a thousand, of ten thousand, and one without end."""
    return _torch().tensor([-(2.0 ** (-10.0 * h / (H - 3))) for h in range(H - 2)] + [-1e-4, 0.0], dtype=_torch().float32, device="cuda")


def _heads(x, heads):
    return None if x is None else to_host(x[:, heads].contiguous()).astype(np.float64)


def _check(got, ref, mag, rows, N, d, dtype, what, state=False):
    """`got` of the heads that the oracle has; rows behind a sequence hold the 7 that was there."""
    if rows is not None:
        assert (got[~rows] == 7.0).all(), f"{what}: rows behind a sequence were written"
        got, ref, mag = (np.where(rows, x, 0.0) for x in (got, ref, mag))
    rest = (N + 2 * d + 65) * E
    tol = rest * mag if dtype == "f32" or state else U * np.abs(ref) + (3 * U * U + rest) * mag
    bad = ~(np.abs(got - ref) <= tol + 1e-37)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound"
    most = 3e-6 if dtype == "f32" or state else U / np.sqrt(3)
    for h in range(ref.shape[1]):
        assert metrics.rel_l2(got[:, h], ref[:, h]) <= most, (what, h, metrics.rel_l2(got[:, h], ref[:, h]))


def _setup(case, seed, count):
    B, H, N, d, dtype, layout, lengths, state = case
    heads = [0, H // 2, H - 2, H - 1]
    n = np.full(B, N) if lengths is None else np.asarray(lengths)
    rows = np.broadcast_to((np.arange(N)[None, :] < n[:, None])[:, None, :, None], (B, len(heads), N, d))
    states = [_states(seed + i, B, H, d, d) if state else None for i in (1, 2)]
    return _draw(seed, B, H, N, d, dtype, layout, count), _decays(H), heads, rows, states


@pytest.mark.parametrize("case", PROMPTS, ids=_id)
def test_prompt(case):
    torch = _torch()
    B, H, N, d, dtype, layout, lengths, state = case
    say(f"decay long prompt {_id(case)}")
    (q, k, v), g, heads, rows, (s_in, _) = _setup(case, 141, 3)
    ref, mag = orc.forward_in_chunks(*(_heads(x, heads) for x in (q, k, v)), to_host(g[heads]), 0.3, _heads(s_in, heads), lengths)
    o, s = _prompt(q, k, v, g, lengths, 0.3, s_in, o=_like(q, 7.0))
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(s).all())
    _check(_heads(o, heads), ref["o"], mag["o"], rows, N, d, dtype, "o")
    _check(_heads(s, heads), ref["s_out"], mag["s_out"], None, N, d, dtype, "s_out", state=True)


@pytest.mark.parametrize("case", BACKWARDS, ids=_id)
def test_backward(case):
    torch = _torch()
    B, H, N, d, dtype, layout, lengths, state = case
    say(f"decay long backward {_id(case)}")
    (q, k, v, do), g, heads, rows, (s_in, ds_out) = _setup(case, 151, 4)
    ref, mag = orc.backward_in_chunks(*(_heads(x, heads) for x in (q, k, v, do)), to_host(g[heads]), -0.4, _heads(s_in, heads), _heads(ds_out, heads), lengths)
    got = _backward(q, k, v, do, g, lengths, -0.4, s_in, ds_out)
    assert all(bool(torch.isfinite(x).all()) for x in got.values())
    for n in ("dq", "dk", "dv"):
        _check(_heads(got[n], heads), ref[n], mag[n], rows, N, d, dtype, n)
    _check(_heads(got["ds_in"], heads), ref["ds_in"], mag["ds_in"], None, N, d, dtype, "ds_in", state=True)
