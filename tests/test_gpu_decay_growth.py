"""Decayed linear attention with l > 1: what is finite by the formulas is so in the results, whatever l^n would be for rows in front of a sequence.

Bounds as in test_gpu_decay.py; a term that passes through n powers counts (1 + n log_decay) times there, so that e^85 is covered as e^-85 is."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import decay_oracle as orc
from tests.gpu_util import say, to_host
from tests.test_gpu_decay import _backward, _check, _draw, _host, _prompt, _states, _torch

pytestmark = pytest.mark.gpu


def _small(xs):
    """Values small enough for products of three of them and e^86 to stay below the largest number of either type."""
    return [x.mul_(2.0 ** -6) for x in xs]


CASES = [   # N, lengths, growth over the sequence (log of the largest power)
    (1, None, 80.0), (2, None, 80.0), (40, None, 80.0), (40, [40, 7, 0], 60.0), (63, None, 86.0), (64, None, 86.0), (70, [70, 33, 1], 86.0),
    (850, None, 86.0), (850, [850, 300, 850], 86.0),
]


@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "bf16"), (112, "bf16"), (128, "bf16"), (32, "f32"), (64, "f32"), (128, "f32")])
@pytest.mark.parametrize("N,lengths,growth", CASES, ids=[f"N{c[0]}{'-ragged' if c[1] else ''}" for c in CASES])
def test_growing_heads(N, lengths, growth, d, dtype):
    """Two heads that grow, one of them slowly, beside one that forgets."""
    torch = _torch()
    B, H, scale = 3, 3, -1.5
    say(f"decay growth N={N} d={d} {dtype}")
    q, k, v, do = _small(_draw(121, B, H, N, d, dtype, "bnhd", 4))
    s_in, ds_out = (x * 2.0 ** -6 for x in (_states(17, B, H, d, d), _states(18, B, H, d, d)))
    g = torch.tensor([growth / N, 0.01, -0.5], device="cuda")
    host = [_host(x) for x in (q, k, v)]
    keep = np.arange(N)[None, :] < np.full(B, N)[:, None] if lengths is None else np.arange(N)[None, :] < np.asarray(lengths)[:, None]
    ref, mag = orc.forward(*host, _host(g), scale, _host(s_in), lengths)
    rows = np.broadcast_to(keep[:, None, :, None], ref["o"].shape)
    o, s = _prompt(q, k, v, g, lengths, scale, s_in)
    _check(o, np.where(rows, ref["o"], 7.0), np.where(rows, mag["o"], 0.0), N, d, dtype, "o", random=False)
    _check(s, ref["s_out"], mag["s_out"], N, d, dtype, "s_out", state=True, random=False)
    ref, mag = orc.backward(*host, _host(do), _host(g), scale, _host(s_in), _host(ds_out), lengths)
    got = _backward(q, k, v, do, g, lengths, scale, s_in, ds_out)
    for n in ("dq", "dk", "dv"):
        _check(got[n], np.where(rows, ref[n], 7.0), np.where(rows, mag[n], 0.0), N, d, dtype, n, random=False)
    _check(got["ds_in"], ref["ds_in"], mag["ds_in"], N, d, dtype, "ds_in", state=True, random=False)


@pytest.mark.parametrize("d", [32, 64, 112, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_grown_is_nothing(d, dtype):
    """l past the largest number: a first token from a state of nothing is k v^T, in a prompt and as a token."""
    torch = _torch()
    B, H = 2, 3
    say(f"decay growth of nothing d={d} {dtype}")
    q, k, v = _draw(122, B, H, 1, d, dtype, "bnhd", 3)
    g = torch.tensor([100.0, 1e30, -0.5], device="cuda")
    want = _host(k)[:, :, 0, :, None] * _host(v)[:, :, 0, None, :]
    for s_in in (None, torch.zeros((B, H, d, d), device="cuda")):
        o, s = _prompt(q, k, v, g, None, 1.0, s_in)
        assert np.abs(_host(s) - want).max() <= 2.0 ** -22 * np.abs(want).max() and np.isfinite(to_host(o)).all()
    pool, o2 = torch.zeros((B, H, d, d), device="cuda"), torch.empty_like(q)
    sv.sv_decay_linattn_token(q, k, v, sv.desc_of(q), g, None, B, 1.0, pool, pool, o2, sv.desc_of(o2))
    torch.cuda.synchronize()
    assert np.array_equal(_host(pool), want.astype(np.float32)) and np.abs(to_host(o2) - to_host(o)).max() <= 2.0 ** -7 * np.abs(to_host(o)).max()
