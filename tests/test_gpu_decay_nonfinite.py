"""Decayed linear attention with NaN and infinities among its tokens: what the formulas make of them, and nothing else.

The oracle (float64, token by token) works on the same tokens: a result that is finite there has to be within test_gpu_decay.py's bounds, one
that is not has to be NaN or infinite."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import decay_oracle as orc
from tests.gpu_util import say, to_host
from tests.test_gpu_decay import E, U, _backward, _draw, _host, _like, _prompt, _space, _states, _torch

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _check(got, ref, mag, N, d, dtype, what, state=False):
    got = to_host(got).astype(np.float64)
    there = np.isfinite(ref)
    assert (np.isfinite(got) == there).all(), f"{what}: {(np.isfinite(got) & ~there).sum()} finite, {(~np.isfinite(got) & there).sum()} not, that should be the other way"
    rest = (N + 2 * d + 65) * E
    tol = rest * mag if dtype == "f32" or state else U * np.abs(ref) + (3 * U * U + rest) * mag
    with np.errstate(invalid="ignore"):
        bad = there & ~(np.abs(got - ref) <= tol + 1e-37)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound"


CASES = [   # B, H, N, lengths: one chunk, chunks of several segments, several chunks of one segment
    (1, 3, 50, None), (2, 3, 301, [301, 222]), (1, 60, 130, None),
]


@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "bf16"), (112, "bf16"), (128, "bf16"), (32, "f32"), (64, "f32"), (112, "f32"), (128, "f32")])
@pytest.mark.parametrize("B,H,N,lengths", CASES, ids=[f"BH{c[0] * c[1]}-N{c[2]}" for c in CASES])
def test_only_what_depends_on_it(B, H, N, lengths, d, dtype):
    torch = _torch()
    say(f"decay nonfinite BH={B * H} N={N} d={d} {dtype}")
    q, k, v, do = _draw(131, B, H, N, d, dtype, "bnhd", 4)
    s_in, ds_out = _states(19, B, H, d, d), _states(20, B, H, d, d)
    g = torch.tensor([-(2.0 ** (-3.0 - h % 5)) for h in range(H)], device="cuda")
    # (tensor, head, token, feature, value); the other heads stay as they are
    at = N // 2
    for x, h, t, f, value in ((v, 0, at, 5, NAN), (v, 0, at + 9, d - 1, INF), (k, 1, at + 3, 17, -INF), (do, 1, at - 7, 2, INF), (q, 2, at + 1, d - 2, NAN)):
        x[0, h, t, f] = value
    n = np.full(B, N) if lengths is None else np.asarray(lengths)
    rows = np.broadcast_to((np.arange(N)[None, :] < n[:, None])[:, None, :, None], q.shape)
    host = [_host(x) for x in (q, k, v)]
    with np.errstate(invalid="ignore"):
        ref, mag = orc.forward(*host, _host(g), 0.3, _host(s_in), lengths)
        back, back_mag = orc.backward(*host, _host(do), _host(g), 0.3, _host(s_in), _host(ds_out), lengths)
    assert np.isfinite(ref["o"]).mean() > 0.5 and (B * H > 6 or not np.isfinite(ref["o"]).all())
    o, s = _prompt(q, k, v, g, lengths, 0.3, s_in)
    _check(o, np.where(rows, ref["o"], 7.0), np.where(rows, mag["o"], 0.0), N, d, dtype, "o")
    _check(s, ref["s_out"], mag["s_out"], N, d, dtype, "s_out", state=True)
    carried = s_in.clone()
    o2, _ = _prompt(q, k, v, g, lengths, 0.3, carried, s_out=carried)
    assert np.array_equal(to_host(o2), to_host(o), equal_nan=True) and np.array_equal(to_host(carried), to_host(s), equal_nan=True)
    got = _backward(q, k, v, do, g, lengths, 0.3, s_in, ds_out)
    for name in ("dq", "dk", "dv"):
        _check(got[name], np.where(rows, back[name], 7.0), np.where(rows, back_mag[name], 0.0), N, d, dtype, name)
    _check(got["ds_in"], back["ds_in"], back_mag["ds_in"], N, d, dtype, "ds_in", state=True)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (112, "bf16"), (64, "f32"), (128, "f32")])
def test_a_state_that_is_no_number(d, dtype):
    """A NaN in the first state of one head stays in that head, and in its column; a sequence of no tokens hands it on as it is."""
    torch = _torch()
    B, H, N, lengths = 2, 2, 150, [150, 0]
    say(f"decay nonfinite state d={d} {dtype}")
    q, k, v = _draw(132, B, H, N, d, dtype, "bhnd", 3)
    s_in = _states(21, B, H, d, d)
    s_in[:, 1, 3, 7] = NAN
    g = torch.tensor([-0.1, -0.01], device="cuda")
    with np.errstate(invalid="ignore"):
        ref, mag = orc.forward(*(_host(x) for x in (q, k, v, g)), 0.3, _host(s_in), lengths)
    o, s = _prompt(q, k, v, g, lengths, 0.3, s_in)
    _check(o[:1], ref["o"][:1], mag["o"][:1], N, d, dtype, "o")
    _check(s, ref["s_out"], mag["s_out"], N, d, dtype, "s_out", state=True)
    assert np.array_equal(to_host(s[1]), to_host(s_in[1]), equal_nan=True) and (to_host(o[1]) == 7.0).all()


def test_nonfinite_tokens_in_a_captured_call():
    """Replayed on clean tokens, on tokens with a NaN and on clean ones again, against eager calls."""
    torch = _torch()
    B, H, N, d = 1, 5, 200, 64
    say("decay nonfinite captured")
    q, k, v = _draw(133, B, H, N, d, "bf16", "bhnd", 3)
    clean = v.clone()
    g, ws = torch.full((H,), -0.02, device="cuda"), _space(sv.sv_decay_linattn_workspace_bytes(B, H, N, d))
    o, s = _like(q, 7.0), torch.zeros((B, H, d, d), device="cuda")

    def call(stream=None):
        sv.sv_decay_linattn(q, k, v, sv.desc_of(q), g, None, 0.5, None, s, o, sv.desc_of(o), ws, stream=stream)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream())
    for poison in (None, (2, 100, 3), None, (4, 0, 63), (0, 199, 0)):
        v.copy_(clean)
        if poison:
            v[0, poison[0], poison[1], poison[2]] = NAN
        call()
        torch.cuda.synchronize()
        want = [to_host(o), to_host(s)]
        o.fill_(7.0)
        s.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(to_host(o), want[0], equal_nan=True) and np.array_equal(to_host(s), want[1], equal_nan=True)
        assert np.isfinite(want[0]).all() == (poison is None)
