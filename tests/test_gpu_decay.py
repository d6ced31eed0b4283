"""Decayed causal linear attention (sv_decay_linattn, its token form and its backward pass) against the float64 recurrences.

How far results may be off, with u = 2^-8 (half a step of bf16), e = 2^-24 and M the sum of the magnitudes of a result's terms, each
counted (1 + n |log_decay|) times for the n decays it passed through (oracle/decay_oracle.py):

  fp32    sums of at most N tokens, d features and a state, in any order, of products rounded a few times: (N + 2 d + 64) e M.
  bf16    the same; states are built up from three bf16 pieces, u^3 = e: one more rounding of each product; what outputs come from enters
          and leaves the state in two, each product off by u^2 = 2^-16 at most: 2 u^2 M; the weighted scores are rounded once, u M at
          most (N <= 64: in two pieces, u^2 M), and the output once, u |o|.

For random data the roundings are independent, so that in the 2-norm over many elements those of scores and outputs come to at most
u / sqrt 3 each, sqrt 2 / sqrt 3 u = 3.2e-3 together, u / sqrt 3 = 2.26e-3 where only the output is rounded."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import decay_oracle as orc
from sv_workloads import metrics
from tests.gpu_util import say, to_host

pytestmark = pytest.mark.gpu

U, E = 2.0 ** -8, 2.0 ** -24


def _torch():
    import torch
    return torch


def _dtype(name):
    return _torch().bfloat16 if name == "bf16" else _torch().float32


def _draw(seed, B, H, N, d, dtype, layout, count):
    """Token tensors [B][H][N][d] of N(0, 1): heads outside tokens, a projection's output, or views of one that holds all of them."""
    torch = _torch()
    gen = torch.Generator().manual_seed(seed)
    if layout == "packed":
        x = torch.randn((B, N, count, H, d), generator=gen).to(_dtype(dtype)).cuda()
        return [x[:, :, i].permute(0, 2, 1, 3) for i in range(count)]
    shape = (B, H, N, d) if layout == "bhnd" else (B, N, H, d)
    xs = [torch.randn(shape, generator=gen).to(_dtype(dtype)).cuda() for _ in range(count)]
    return xs if layout == "bhnd" else [x.permute(0, 2, 1, 3) for x in xs]


def _like(x, value):
    """A tensor with x's strides, filled."""
    torch = _torch()
    y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    return y.fill_(value)


def _decays(H, kind="mixed"):
    g = {"mixed": [-(2.0 ** (-10.0 * h / max(1, H - 1))) for h in range(H)],
         "edge": [[0.0, float("-inf"), -1e-6, -3.0, -50.0, -1e30][h % 6] for h in range(H)]}[kind]
    return _torch().tensor(g, dtype=_torch().float32, device="cuda")


def _space(nbytes):
    assert nbytes > 0
    return _torch().empty(nbytes, dtype=_torch().uint8, device="cuda").fill_(255)       # NaNs: nothing of it may be used as it is


def _ints(x):
    return None if x is None else _torch().tensor(x, dtype=_torch().int32, device="cuda")


def _states(seed, *shape):
    torch = _torch()
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def _host(x):
    return None if x is None else to_host(x).astype(np.float64)


def _check(got, ref, mag, N, d, dtype, what, state=False, random=True):
    got = _host(got)
    rest = (N + 2 * d + 64) * E
    if dtype == "f32" or state:
        tol = (rest + E) * mag
    else:
        tol = U * np.abs(ref) + ((U if N > 64 else U * U) + 2 * U * U + rest) * mag
    bad = ~(np.abs(got - ref) <= tol + 1e-37)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound, worst by {np.nanmax((np.abs(got - ref) - tol)[bad])}"
    if random and got.size >= 2048:
        most = 3e-6 if dtype == "f32" or state else 3.5e-3 if N > 64 else 2.3e-3
        assert metrics.rel_l2(got, ref) <= most, f"{what}: {metrics.rel_l2(got, ref)}"


def _prompt(q, k, v, g, lengths, scale, s_in, want_state=True, o=None, s_out=None, stream=None):
    torch = _torch()
    B, H, N, d = q.shape
    o = _like(q, 7.0) if o is None else o
    s_out = torch.full((B, H, d, d), 7.0, device="cuda") if s_out is None and want_state else s_out
    ws = _space(sv.sv_decay_linattn_workspace_bytes(B, H, N, d))
    sv.sv_decay_linattn(q, k, v, sv.desc_of(q), g, _ints(lengths), scale, s_in, s_out, o, sv.desc_of(o), ws, stream=stream)
    torch.cuda.synchronize()
    return o, s_out


def _backward(q, k, v, do, g, lengths, scale, s_in, ds_out):
    torch = _torch()
    B, H, N, d = q.shape
    dq, dk, dv = (_like(q, 7.0) for _ in range(3))
    ds_in = torch.full((B, H, d, d), 7.0, device="cuda")
    ws = _space(sv.sv_decay_linattn_backward_workspace_bytes(B, H, N, d))
    sv.sv_decay_linattn_backward(q, k, v, sv.desc_of(q), do, sv.desc_of(do), g, _ints(lengths), scale, s_in, ds_out, dq, dk, dv, ds_in, ws)
    torch.cuda.synchronize()
    return {"dq": dq, "dk": dk, "dv": dv, "ds_in": ds_in}


CASES = [   # B, H, N, d, dtype, layout, lengths, state, decays
    (1, 2, 1, 64, "bf16", "bhnd", None, True, "mixed"),
    (1, 3, 2, 32, "f32", "bnhd", None, False, "mixed"),
    (2, 2, 31, 112, "bf16", "packed", None, True, "mixed"),
    (1, 2, 32, 128, "f32", "bhnd", None, True, "mixed"),
    (1, 2, 33, 128, "bf16", "bnhd", None, True, "mixed"),
    (1, 6, 63, 32, "bf16", "bhnd", None, True, "edge"),
    (1, 6, 64, 64, "bf16", "packed", None, True, "edge"),
    (2, 6, 65, 112, "f32", "packed", None, True, "edge"),
    (1, 2, 127, 112, "bf16", "bhnd", None, False, "mixed"),
    (1, 2, 129, 128, "bf16", "packed", None, True, "mixed"),
    (1, 3, 700, 64, "bf16", "bhnd", None, True, "mixed"),            # several segments of chunks
    (2, 2, 517, 128, "f32", "bnhd", None, True, "mixed"),
    (1, 6, 1000, 32, "f32", "bhnd", None, True, "edge"),
    (1, 6, 777, 112, "bf16", "packed", None, True, "edge"),
    (6, 2, 449, 64, "bf16", "bnhd", [449, 0, 1, 64, 385, 200], True, "mixed"),     # lengths that end in every place of a segment
    (5, 2, 321, 128, "bf16", "packed", [65, 320, 0, 5000, -3], True, "mixed"),     # held to [0, N]
    (4, 3, 230, 112, "f32", "packed", [129, 1, 0, 97], False, "mixed"),
    (13, 40, 200, 32, "bf16", "bhnd", None, True, "mixed"),          # one workgroup per head
    (2, 32, 3000, 32, "bf16", "bnhd", [3000, 1777], True, "mixed"),  # segments of several chunks, whose first ones weigh nothing for some heads
    (1, 40, 1500, 32, "f32", "bhnd", None, True, "mixed"),
    (1, 60, 1200, 64, "bf16", "bhnd", None, True, "edge"),
    (9, 60, 67, 64, "f32", "bnhd", [67, 3, 0, 66, 32, 33, 1, 64, 65], True, "mixed"),
]


def _id(c):
    return f"B{c[0]}H{c[1]}N{c[2]}d{c[3]}-{c[4]}-{c[5]}{'-ragged' if c[6] else ''}{'' if c[7] else '-nostate'}-{c[8]}"


def _behind(x, lengths, value):
    """Fills the rows behind the sequences' lengths; returns which rows are tokens."""
    B, H, N, d = x.shape
    n = np.clip(np.full(B, N) if lengths is None else np.asarray(lengths), 0, N)
    for b in range(B):
        x[b, :, n[b]:] = value
    return np.arange(N)[None, :] < n[:, None]


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_prompt(case):
    B, H, N, d, dtype, layout, lengths, state, decays = case
    say(f"decay prompt {_id(case)}")
    q, k, v = _draw(11, B, H, N, d, dtype, layout, 3)
    g, scale = _decays(H, decays), 0.3
    s_in = _states(5, B, H, d, d) if state else None
    keep = _behind(q, lengths, 0.0)
    ref, mag = orc.forward(_host(q), _host(k), _host(v), _host(g), scale, _host(s_in), lengths)
    for x in (q, k, v):
        _behind(x, lengths, float("nan"))                     # nothing behind a sequence may be read
    o, s_out = _prompt(q, k, v, g, lengths, scale, s_in)
    rows = np.broadcast_to(keep[:, None, :, None], ref["o"].shape)
    got = to_host(o)
    assert (got[~rows] == 7.0).all(), "rows behind a sequence were written"
    _check(o, np.where(rows, ref["o"], 7.0), np.where(rows, mag["o"], 0.0), N, d, dtype, "o")
    _check(s_out, ref["s_out"], mag["s_out"], N, d, dtype, "s_out", state=True)
    # without the final state, and with it in place of the first
    o2, _ = _prompt(q, k, v, g, lengths, scale, s_in, want_state=False)
    assert np.array_equal(to_host(o2), got)
    if state:
        carried = s_in.clone()
        o3, _ = _prompt(q, k, v, g, lengths, scale, carried, s_out=carried)
        assert np.array_equal(to_host(o3), got) and _torch().equal(carried, s_out)


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_backward(case):
    B, H, N, d, dtype, layout, lengths, state, decays = case
    say(f"decay backward {_id(case)}")
    q, k, v = _draw(21, B, H, N, d, dtype, layout, 3)
    do, = _draw(22, B, H, N, d, dtype, "bnhd" if layout == "packed" else layout, 1)
    g, scale = _decays(H, decays), -0.4
    s_in, ds_out = (_states(6, B, H, d, d), _states(7, B, H, d, d)) if state else (None, None)
    keep = _behind(q, lengths, 0.0)
    ref, mag = orc.backward(*(_host(x) for x in (q, k, v, do, g)), scale, _host(s_in), _host(ds_out), lengths)
    for x in (q, k, v, do):
        _behind(x, lengths, float("nan"))
    got = _backward(q, k, v, do, g, lengths, scale, s_in, ds_out)
    rows = np.broadcast_to(keep[:, None, :, None], ref["dq"].shape)
    for n in ("dq", "dk", "dv"):
        assert (to_host(got[n])[~rows] == 7.0).all(), f"{n}: rows behind a sequence were written"
        _check(got[n], np.where(rows, ref[n], 7.0), np.where(rows, mag[n], 0.0), N, d, dtype, n)
    _check(got["ds_in"], ref["ds_in"], mag["ds_in"], N, d, dtype, "ds_in", state=True)


def test_gradients_are_those_of_the_forward_call():
    """Central differences of sum(o do) + sum(s_out ds_out) in fp32, along random directions: the loss is bilinear in each input, so
    the difference quotient is exact but for rounding, 2 x the sum of magnitudes x (N + 2 d + 64) 2^-24 over the step of 1."""
    torch = _torch()
    B, H, N, d, scale = 2, 3, 97, 32, 0.5
    lengths = [97, 40]
    q, k, v = _draw(31, B, H, N, d, "f32", "bhnd", 3)
    do, = _draw(32, B, H, N, d, "f32", "bhnd", 1)
    s_in, ds_out = _states(8, B, H, d, d), _states(9, B, H, d, d)
    g = _decays(H)
    for x in (q, k, v, do):
        _behind(x, lengths, 0.0)
    say("decay backward against differences")
    grads = _backward(q, k, v, do, g, lengths, scale, s_in, ds_out)

    def loss(q, k, v, s_in):
        o = torch.zeros_like(q)
        o, s = _prompt(q, k, v, g, lengths, scale, s_in, o=o)
        return float((o.double() * do.double()).sum() + (s.double() * ds_out.double()).sum())

    for name, at in (("dq", 0), ("dk", 1), ("dv", 2), ("ds_in", 3)):
        args = [q, k, v, s_in]
        step = torch.randn(args[at].shape, generator=torch.Generator().manual_seed(40 + at)).cuda()
        if at < 3:
            _behind(step, lengths, 0.0)
        there = [a + step if i == at else a for i, a in enumerate(args)]
        back = [a - step if i == at else a for i, a in enumerate(args)]
        slope = (loss(*there) - loss(*back)) / 2
        grad = torch.where(torch.isfinite(grads[name]), grads[name], 0.0)
        if at < 3:
            _behind(grad, lengths, 0.0)
        want = float((grad.double() * step.double()).sum())
        # magnitude of the loss: every o (do) and s_out (ds_out) term
        ref, mag = orc.forward(*(np.abs(_host(x)) for x in there[:3]), _host(g), abs(scale), np.abs(_host(there[3])), lengths)
        size = (mag["o"] * np.abs(_host(do))).sum() + (mag["s_out"] * np.abs(_host(ds_out))).sum()
        assert abs(slope - want) <= 2 * size * (N + 2 * d + 64) * E, (name, slope, want)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (112, "bf16"), (128, "f32"), (32, "f32")])
def test_prompt_continues_where_the_last_one_ended(d, dtype):
    """Cut anywhere, the two parts give what the whole gives: a sequence's tokens and state do not depend on the cut."""
    torch = _torch()
    B, H, N, cut, scale = 1, 4, 420, 133, 0.25
    say(f"decay prompt in two parts d={d} {dtype}")
    q, k, v = _draw(51, B, H, N, d, dtype, "bnhd", 3)
    g = _decays(H)
    ref, mag = orc.forward(*(_host(x) for x in (q, k, v, g)), scale)
    o1, s1 = _prompt(*(x[:, :, :cut] for x in (q, k, v)), g, None, scale, None)
    o2, s2 = _prompt(*(x[:, :, cut:] for x in (q, k, v)), g, None, scale, s1)
    _check(torch.cat([o1, o2], dim=2), ref["o"], mag["o"], N, d, dtype, "o")
    _check(s2, ref["s_out"], 2 * mag["s_out"], N, d, dtype, "s_out", state=True)


@pytest.mark.parametrize("d", [32, 64, 112, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,pool,H", [(1, 1, 2), (5, 9, 3), (70, 80, 5)])
def test_token(d, dtype, rows, pool, H):
    """Slots in any order, idle rows among them, a slot named twice; other slots and idle rows stay as they were.  Bound: two roundings per
    element of the state, d + 2 of the output's sum, and the output's own."""
    torch = _torch()
    say(f"decay token d={d} {dtype} rows={rows} pool={pool} H={H}")
    q, k, v = _draw(61, rows, H, 1, d, dtype, "packed", 3)
    g, scale = _decays(H), 0.3
    S = _states(12, pool, H, d, d)
    slots = list(np.random.default_rng(3).permutation(pool)[:rows])
    serves = list(range(rows))
    if rows >= 5:
        slots[1], slots[3], slots[4] = -1, pool, slots[0]            # idle, idle, and named by row 0 already
        serves = [r for r in serves if r not in (1, 3, 4)]
    for in_place in (False, True):
        s_in = S.clone()
        s_out = s_in if in_place else torch.full_like(S, 7.0)
        o = _like(q, 7.0)
        sv.sv_decay_linattn_token(q, k, v, sv.desc_of(q), g, _ints(slots), pool, scale, s_in, s_out, o, sv.desc_of(o))
        torch.cuda.synchronize()
        before, got_s, got_o = _host(S), _host(s_out), _host(o)
        qh, kh, vh, l = _host(q), _host(k), _host(v), np.exp(_host(g))[:, None, None]
        touched = np.zeros(pool, dtype=bool)
        for r in serves:
            s, touched[slots[r]] = slots[r], True
            want = l * before[s] + kh[r, :, 0, :, None] * vh[r, :, 0, None, :]
            size = l * np.abs(before[s]) + np.abs(kh[r, :, 0, :, None] * vh[r, :, 0, None, :])
            assert (np.abs(got_s[s] - want) <= 4 * E * size).all()
            out = scale * (qh[r, :, 0, :, None] * want).sum(1)
            mag = scale * (np.abs(qh[r, :, 0, :, None]) * size).sum(1)
            u = U if dtype == "bf16" else E
            assert (np.abs(got_o[r, :, 0] - out) <= u * np.abs(out) + (d + 8) * E * mag).all()
        idle = [r for r in range(rows) if r not in serves]
        assert (got_o[idle] == 7.0).all()
        assert np.array_equal(got_s[~touched], before[~touched] if in_place else np.full_like(before[~touched], 7.0))


def test_token_without_slots_follows_a_prompt():
    """A prompt, then tokens one by one, give what the longer prompt gives (fp32 tokens; the sums' bound)."""
    torch = _torch()
    B, H, N, more, d, scale = 3, 4, 70, 5, 64, 0.25
    say("decay tokens after a prompt")
    q, k, v = _draw(71, B, H, N + more, d, "f32", "bhnd", 3)
    g = _decays(H)
    ref, mag = orc.forward(*(_host(x) for x in (q, k, v, g)), scale)
    _, S = _prompt(*(x[:, :, :N] for x in (q, k, v)), g, None, scale, None)
    for t in range(N, N + more):
        one = [x[:, :, t:t + 1] for x in (q, k, v)]
        o = torch.full((B, H, 1, d), 7.0, device="cuda")
        sv.sv_decay_linattn_token(*one, sv.desc_of(one[0]), g, None, B, scale, S, S, o, sv.desc_of(o))
        torch.cuda.synchronize()
        _check(o, ref["o"][:, :, t:t + 1], mag["o"][:, :, t:t + 1], N + more, d, "f32", f"token {t}", random=False)
    _check(S, ref["s_out"], mag["s_out"], N + more, d, "f32", "state", state=True)


def test_long_memory_over_many_chunks():
    """One workgroup per head over 300 chunks with a decay at or just below 1.  fp32 tokens that are all ones in feature 0: S[0][0] is the
    geometric sum.  Its bound: the matrix instructions add two tokens at a time to the state itself, N / 2 roundings of a sum that only
    grows, and each of the N / 32 chunks multiplies it once (two roundings); 64 for the weights."""
    torch = _torch()
    B, H, N, d = 130, 4, 9600, 32
    say("decay long memory")
    k = torch.zeros((B, H, N, d), device="cuda")
    k[..., 0] = 1.0
    g = torch.tensor([0.0, -1e-7, -1.2345e-5, -1e-3], device="cuda")
    _, s = _prompt(k, k, k, g, None, 1.0, None)
    l = np.exp(_host(g))
    want = np.array([N if x == 1.0 else (1 - x ** N) / (1 - x) for x in l])
    got = _host(s)
    assert (np.abs(got[:, :, 0, 0] - want) <= (N / 2 + 2 * N / 32 + 64) * E * want).all(), (got[0, :, 0, 0], want)
    got[:, :, 0, 0] = 0.0
    assert (got == 0.0).all()


def test_old_tokens_lose_nothing_but_their_decay():
    """A first token and 9 599 empty ones behind it: the state is l^{N-1} k v^T, through 300 multiplications by l^C, which is held as two
    floats: one rounding of the state for each chunk (2^-24 at most, and near l = 1 all in the same direction: the state falls by nearly the
    same number of steps each time), so 300 x 2^-24 and 8 for the first weights."""
    torch = _torch()
    B, H, N, d = 130, 4, 9600, 32
    say("decay old tokens")
    k, v = torch.zeros((B, H, N, d), device="cuda"), torch.zeros((B, H, N, d), device="cuda")
    k[:, :, 0, 0] = 1.0
    v[:, :, 0] = _states(14, B, H, d)
    g = torch.tensor([-3e-7, -1.7e-6, -1.2345e-5, -1e-4], device="cuda")
    _, s = _prompt(k, k, v, g, None, 1.0, None)
    want = np.exp(_host(g) * (N - 1))[None, :, None] * _host(v)[:, :, 0]
    got = _host(s)[:, :, 0]
    assert (np.abs(got - want) <= (N / 32 + 8) * E * np.abs(want)).all()


def test_nothing_outside_the_buffers_is_touched():
    """Outputs, states and workspace between guard areas; inputs end where their memory ends."""
    torch = _torch()
    B, H, N, d = 2, 3, 203, 112
    say("decay guards")
    q, k, v, do = _draw(81, B, H, N, d, "bf16", "bhnd", 4)
    g, lengths = _decays(H), _ints([203, 77])
    guard = 4096

    def fenced(nbytes):
        whole = torch.full((nbytes + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
        return whole, whole[guard:guard + nbytes]

    def clean(whole):
        return bool((whole[:guard] == 0xA5).all()) and bool((whole[-guard:] == 0xA5).all())
    tok, st = B * H * N * d * 2, B * H * d * d * 4
    fences, views = [], []
    for n in (tok, tok, tok, tok, st, st, sv.sv_decay_linattn_workspace_bytes(B, H, N, d), sv.sv_decay_linattn_backward_workspace_bytes(B, H, N, d)):
        w, view = fenced(n)
        fences.append(w)
        views.append(view)
    o, dq, dk, dv = (x.view(torch.bfloat16).view(B, H, N, d) for x in views[:4])
    s_out, ds_in = (x.view(torch.float32).view(B, H, d, d) for x in views[4:6])
    sv.sv_decay_linattn(q, k, v, sv.desc_of(q), g, lengths, 1.0, None, s_out, o, sv.desc_of(o), views[6])
    sv.sv_decay_linattn_backward(q, k, v, sv.desc_of(q), do, sv.desc_of(do), g, lengths, 1.0, None, s_out, dq, dk, dv, ds_in, views[7])
    sv.sv_decay_linattn_token(*(x[:, :, :1] for x in (q, k, v)), sv.desc_of(q[:, :, :1]), g, None, B, 1.0, s_out, ds_in, o[:, :, :1],
                              sv.desc_of(o[:, :, :1]))
    torch.cuda.synchronize()
    assert all(clean(w) for w in fences)


def test_repeatable_and_captured():
    """Two calls give the same bits, on another stream too; a captured prompt, token and backward pass replays on new contents of the
    same buffers (lengths and slots among them), with eager work between the replays."""
    torch = _torch()
    B, H, N, d, scale = 2, 5, 300, 64, 0.3
    say("decay capture")
    dev = [torch.empty((B, H, N, d), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    q, k, v, do = dev
    g, lengths, slots = _decays(H), _ints([N, N]), _ints([0, 1])
    one = [x[:, :, :1] for x in (q, k, v)]
    ws = _space(sv.sv_decay_linattn_workspace_bytes(B, H, N, d))
    wb = _space(sv.sv_decay_linattn_backward_workspace_bytes(B, H, N, d))

    def buffers():
        outs = [torch.full_like(q, 7.0) for _ in range(4)] + [torch.full((B, H, d, d), 7.0, device="cuda") for _ in range(3)]
        return outs + [torch.full((B, H, 1, d), 7.0, dtype=torch.bfloat16, device="cuda")]

    def enqueue(out, stream):
        o, dq, dk, dv, s_out, ds_in, pool, ot = out
        sv.sv_decay_linattn(q, k, v, sv.desc_of(q), g, lengths, scale, None, s_out, o, sv.desc_of(o), ws, stream=stream)
        sv.sv_decay_linattn_token(*one, sv.desc_of(one[0]), g, slots, B, scale, s_out, pool, ot, sv.desc_of(ot), stream=stream)
        sv.sv_decay_linattn_backward(q, k, v, sv.desc_of(q), do, sv.desc_of(do), g, lengths, scale, None, s_out, dq, dk, dv, ds_in, wb, stream=stream)

    def fill(seed):
        gen = torch.Generator().manual_seed(seed)
        for x in dev:
            x.copy_(torch.randn(x.shape, generator=gen))
        lengths.copy_(torch.tensor([N, 1 + (seed * 37) % N], dtype=torch.int32))
        slots.copy_(torch.tensor([1, 0] if seed % 2 else [0, -1], dtype=torch.int32))
        torch.cuda.synchronize()
    fill(1)
    other = torch.cuda.Stream()
    a, b, replayed = buffers(), buffers(), buffers()
    torch.cuda.synchronize()
    enqueue(a, None)
    torch.cuda.synchronize()
    enqueue(b, other)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        enqueue(replayed, torch.cuda.current_stream())
    for seed in (2, 3, 4, 5):
        fill(seed)
        eager = buffers()
        enqueue(eager, None)
        torch.cuda.synchronize()
        for x in replayed:
            x.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, replayed)), seed


def test_heads_of_more_than_2_gib():
    """Rows 1.3 MiB apart: a head spans 2.6 GiB, and byte offsets inside it pass 32 bits' sign."""
    torch = _torch()
    N, d, wide = 2100, 64, 655360
    say("decay heads of more than 2 GiB")
    big = torch.empty((N, wide), dtype=torch.bfloat16, device="cuda")
    q, k, v = (big[:, 1000 * 64 * i:1000 * 64 * i + d].unflatten(0, (1, 1, N)) for i in range(3))
    for x, y in zip((q, k, v), _draw(91, 1, 1, N, d, "bf16", "bhnd", 3)):
        x.copy_(y)
    g = _decays(1)
    dense = [x.contiguous() for x in (q, k, v)]
    o, s = _prompt(q, k, v, g, None, 0.5, None, o=torch.full((1, 1, N, d), 7.0, dtype=torch.bfloat16, device="cuda"))
    o2, s2 = _prompt(*dense, g, None, 0.5, None)
    assert torch.equal(o, o2) and torch.equal(s, s2)
    do = dense[1]
    ws = _space(sv.sv_decay_linattn_backward_workspace_bytes(1, 1, N, d))
    grads = [big[:, 1000 * 64 * i:1000 * 64 * i + d].unflatten(0, (1, 1, N)) for i in range(3, 6)]
    sv.sv_decay_linattn_backward(q, k, v, sv.desc_of(q), do, sv.desc_of(do), g, None, 0.5, None, None, *grads, None, ws)
    torch.cuda.synchronize()
    want = _backward(*dense, do, g, None, 0.5, None, None)
    assert all(torch.equal(x, want[n]) for x, n in zip(grads, ("dq", "dk", "dv")))
