"""Layer norm (sv_layernorm) and its backward pass against 64 bits.

Bounds, with e = 2^-24 and u = 2^-8 (bf16) or e (fp32) for the one rounding to the tensors' type.  A lane adds up at most 48 terms of a row
one after the other, the lanes are added in a tree of six steps and at most 16 waves in a row: a row's sum is off by 64 e of its terms'
magnitudes.  So, with A the row's mean magnitude and part = (|x| + A) rstd: mean is off by 64 e A; x - mean by 65 e (|x| + A); the variance by
64 e of itself and twice the mean of |x - mean| 65 e (|x| + A), which is at most var S with S = sqrt(mean part^2) (Cauchy and Schwarz); rstd
by half of that and its own two roundings, less than (64 + 65 S) e of itself; xh by (130 + 65 S) e (|xh| + part).  The backward pass is given
mean and rstd; its sums' terms are off by a few e of the magnitudes that the oracle adds up, 80 e in all.  dw and db: a lane adds up its rows,
at most 64 lanes and 64 + 16 partial sums are added one after the other: rows / 32 + 80 covers every number of rows."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import layer_oracle as orc
from tests.gpu_util import say, to_host

pytestmark = pytest.mark.gpu

U, E = 2.0 ** -8, 2.0 ** -24


def _torch():
    import torch
    return torch


def _rows(seed, B, H, N, d, dtype, layout, shift):
    torch = _torch()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((B, H, N, d), generator=torch.Generator().manual_seed(seed)) + shift
    if layout == "bhnd":
        return x.to(dt).cuda()
    if layout == "bnhd":
        return x.permute(0, 2, 1, 3).contiguous().to(dt).cuda().permute(0, 2, 1, 3)
    wide = torch.full((B, H, N + 3, d + 32), float("nan"), dtype=dt, device="cuda")               # rows apart, tokens left over
    wide[:, :, 1:N + 1, 16:16 + d] = x.to(dt).cuda()
    return wide[:, :, 1:N + 1, 16:16 + d]


def _params(seed, heads, d):
    torch = _torch()
    gen = torch.Generator().manual_seed(seed)
    return (1 + 0.3 * torch.randn((heads, d), generator=gen)).cuda(), (0.2 * torch.randn((heads, d), generator=gen)).cuda()


def _like(x, value):
    return _torch().empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device).fill_(value)


def _space(B, H, N, d):
    return _torch().empty(sv.sv_layernorm_backward_workspace_bytes(B, H, N, d), dtype=_torch().uint8, device="cuda").fill_(255)


WIDTHS_BF16 = [8, 16, 24, 32, 40, 64, 72, 112, 128, 256, 264, 512, 520, 1024, 1504, 2048, 2240, 2568, 3064, 3080, 4096, 4104, 6720, 8192]
WIDTHS_F32 = [4, 12, 16, 28, 36, 64, 112, 128, 132, 252, 260, 512, 1020, 1536, 1540, 2240, 2052, 4096, 4100, 8192]
CASES = [(2, 3, 37, d, "bf16", "bhnd", True, 0.3) for d in WIDTHS_BF16] + [(1, 2, 29, d, "f32", "bnhd", False, 0.3) for d in WIDTHS_F32] + [
    (1, 1, 1, 2240, "bf16", "bhnd", False, 5.0), (1, 1, 1, 32, "f32", "bhnd", True, 0.0), (3, 5, 211, 112, "bf16", "bnhd", True, 5.0),
    (3, 5, 211, 112, "bf16", "bnhd", False, 1.0), (2, 4, 333, 128, "f32", "apart", True, 1.0), (1, 1, 2500, 320, "bf16", "apart", False, 0.3),
    (2, 20, 900, 64, "bf16", "bhnd", False, 0.3), (1, 3, 700, 1504, "f32", "bnhd", True, 0.3), (2, 1500, 3, 32, "bf16", "bnhd", True, 0.3),
]


def _id(c):
    return f"{c[0]}x{c[1]}x{c[2]}x{c[3]}-{c[4]}-{c[5]}{'-heads' if c[6] else ''}"


def _sizes(x, mean, rstd):
    """(|x| + A) rstd per element and S per row."""
    A = np.abs(x).mean(-1, keepdims=True)
    part = (np.abs(x) + A) * rstd[..., None]
    return part, np.sqrt((part ** 2).mean(-1, keepdims=True))


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_forward(case):
    torch = _torch()
    B, H, N, d, dtype, layout, per_head, shift = case
    say(f"norm forward {_id(case)}")
    x = _rows(1, B, H, N, d, dtype, layout, shift)
    heads = H if per_head else 1
    w, b = _params(2, heads, d)
    y = _like(x, 7.0)
    mean, rstd = (torch.full((B, H, N), 7.0, device="cuda") for _ in range(2))
    sv.sv_layernorm(x, sv.desc_of(x), w, b, heads, 1e-5, y, sv.desc_of(y), mean, rstd)
    torch.cuda.synchronize()
    xh = to_host(x).astype(np.float64)
    ref, rm, rr = orc.norm(xh, to_host(w), to_host(b), 1e-5)
    part, S = _sizes(xh, rm, rr)
    assert (np.abs(to_host(mean) - rm) <= 64 * E * np.abs(xh).mean(-1)).all()
    assert (np.abs(to_host(rstd) - rr) <= (64 + 65 * S[..., 0]) * E * rr).all()
    wn = np.abs(np.broadcast_to(to_host(w).astype(np.float64), (H, d)))[None, :, None, :]
    normed = np.abs((xh - rm[..., None]) * rr[..., None])
    u = U if dtype == "bf16" else E
    tol = u * np.abs(ref) + (130 + 65 * S) * E * wn * (normed + part) + 2 * E * np.abs(ref)
    assert (np.abs(to_host(y) - ref) <= tol).all()
    # without statistics and parameters; and in place
    plain = _like(x, 7.0)
    sv.sv_layernorm(x, sv.desc_of(x), None, None, 1, 1e-5, plain, sv.desc_of(plain), None, None)
    ones, zeros = torch.ones((1, d), device="cuda"), torch.zeros((1, d), device="cuda")
    same = _like(x, 7.0)
    sv.sv_layernorm(x, sv.desc_of(x), ones, zeros, 1, 1e-5, same, sv.desc_of(same), None, None)
    torch.cuda.synchronize()
    assert torch.equal(plain, same)
    sv.sv_layernorm(x, sv.desc_of(x), w, b, heads, 1e-5, x, sv.desc_of(x), None, None)
    torch.cuda.synchronize()
    assert torch.equal(x, y)


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_backward(case):
    torch = _torch()
    B, H, N, d, dtype, layout, per_head, shift = case
    say(f"norm backward {_id(case)}")
    x, dy = _rows(1, B, H, N, d, dtype, layout, shift), _rows(3, B, H, N, d, dtype, "bhnd", 0.1)
    heads = H if per_head else 1
    w, _ = _params(2, heads, d)
    _, mean, rstd = orc.norm(to_host(x), None, None, 1e-5)
    mean, rstd = (torch.from_numpy(t.astype(np.float32)).cuda() for t in (mean, rstd))
    dx, dw, db = _like(x, 7.0), torch.full((heads, d), 7.0, device="cuda"), torch.full((heads, d), 7.0, device="cuda")
    ws = _space(B, H, N, d)
    args = (x, sv.desc_of(x), dy, sv.desc_of(dy), w, heads, mean, rstd)
    sv.sv_layernorm_backward(*args, dx, sv.desc_of(dx), dw, db, ws)
    torch.cuda.synchronize()
    ref, mag = orc.norm_backward(to_host(x), to_host(dy), to_host(w), to_host(mean), to_host(rstd), per_head)
    u = U if dtype == "bf16" else E
    assert (np.abs(to_host(dx) - ref["dx"]) <= u * np.abs(ref["dx"]) + 80 * E * mag["dx"]).all()
    c = B * H * N / 32 + 80
    assert (np.abs(to_host(dw) - ref["dw"]) <= c * E * mag["dw"]).all()
    assert (np.abs(to_host(db) - ref["db"]) <= c * E * mag["db"]).all()
    # one of the parameters, none of them, and dx over dy
    dx2, dw2, db2 = _like(x, 7.0), torch.full_like(dw, 7.0), torch.full_like(db, 7.0)
    sv.sv_layernorm_backward(*args, dx2, sv.desc_of(dx2), dw2, None, ws)
    sv.sv_layernorm_backward(*args, dx2, sv.desc_of(dx2), None, db2, ws)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)
    sv.sv_layernorm_backward(*args, dx2.fill_(7.0), sv.desc_of(dx2), None, None, None)
    sv.sv_layernorm_backward(*args, dy, sv.desc_of(dy), None, None, None)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2) and torch.equal(dx, dy)


def test_gradients_are_those_of_the_forward_call():
    """Differences of sum(y g) in fp32 along random directions.  For w and b the loss is linear, the quotient exact but for rounding; for x the
    central difference with a step of h is off by h^2 / 6 times the third derivative: at h = 2^-7 along directions of N(0, 1) entries
    h^2 / 6 is 1.0e-5, and the third derivative of a row's contribution is at most 60 |g| per element for rows of deviation 1."""
    torch = _torch()
    B, H, N, d = 2, 3, 11, 64
    say("norm backward against differences")
    x, g = _rows(1, B, H, N, d, "f32", "bhnd", 0.3), _rows(3, B, H, N, d, "f32", "bhnd", 0.0)
    w, b = _params(2, H, d)
    y = torch.empty_like(x)
    mean, rstd = (torch.empty((B, H, N), device="cuda") for _ in range(2))

    def loss(x, w, b):
        sv.sv_layernorm(x, sv.desc_of(x), w, b, H, 1e-5, y, sv.desc_of(y), mean, rstd)
        torch.cuda.synchronize()
        return float((y.double() * g.double()).sum())
    loss(x, w, b)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    sv.sv_layernorm_backward(x, sv.desc_of(x), g, sv.desc_of(g), w, H, mean, rstd, dx, sv.desc_of(dx), dw, db, _space(B, H, N, d))
    torch.cuda.synchronize()
    rounding = float(g.abs().sum()) * 8 * 400 * E          # |y| < 8; (130 + 65 S) e with S < 4
    for grad, at, h in ((dx, 0, 2.0 ** -7), (dw, 1, 1.0), (db, 2, 1.0)):
        args = [x, w, b]
        step = torch.randn(args[at].shape, generator=torch.Generator().manual_seed(9 + at)).cuda()
        there = [t + h * step if i == at else t for i, t in enumerate(args)]
        back = [t - h * step if i == at else t for i, t in enumerate(args)]
        slope = (loss(*there) - loss(*back)) / (2 * h)
        want = float((grad.double() * step.double()).sum())
        third = h * h / 6 * 60 * float(g.abs().sum()) * 2 if at == 0 else 0.0
        assert abs(slope - want) <= rounding / h + third, (at, slope, want)


def test_guards_and_capture():
    """Nothing outside the buffers is written; a captured forward and backward pass replays on new contents with eager work in between."""
    torch = _torch()
    B, H, N, d, guard = 1, 4, 333, 112, 4096
    say("norm guards, captured")
    x, dy = _rows(1, B, H, N, d, "bf16", "bhnd", 0.3), _rows(3, B, H, N, d, "bf16", "bhnd", 0.0)
    w, b = _params(2, H, d)

    def buffers():
        fences, views = [], []
        for n in (B * H * N * d * 2, B * H * N * d * 2, B * H * N * 4 + 16, B * H * N * 4 + 16, H * d * 4, H * d * 4,
                  sv.sv_layernorm_backward_workspace_bytes(B, H, N, d)):
            whole = torch.full((n + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
            fences.append(whole)
            views.append(whole[guard:guard + n])
        y, dx = (v.view(torch.bfloat16).view(B, H, N, d) for v in views[:2])
        mean, rstd = (v.view(torch.float32)[:B * H * N].view(B, H, N) for v in views[2:4])
        dw, db = (v.view(torch.float32).view(H, d) for v in views[4:6])
        return fences, (y, dx, mean, rstd, dw, db), views[6]

    def enqueue(out, ws, stream):
        y, dx, mean, rstd, dw, db = out
        sv.sv_layernorm(x, sv.desc_of(x), w, b, H, 1e-5, y, sv.desc_of(y), mean, rstd, stream=stream)
        sv.sv_layernorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, H, mean, rstd, dx, sv.desc_of(dx), dw, db, ws, stream=stream)
    fences, captured, ws = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        enqueue(captured, ws, torch.cuda.current_stream())
    for seed in (4, 5, 6):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))
        other, eager, ws2 = buffers()
        enqueue(eager, ws2, torch.cuda.Stream() if seed == 5 else None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(captured, eager))
        for whole in fences + other:
            assert bool((whole[:guard] == 0xA5).all()) and bool((whole[-guard:] == 0xA5).all())


def test_many_rows():
    """More rows than lanes walk at once, of every number of parameter rows; statistics of each where they belong."""
    torch = _torch()
    B, H, N, d = 3, 7, 4001, 32
    say("norm many rows")
    x = _rows(1, B, H, N, d, "f32", "bnhd", 0.3)
    for heads in (1, H):
        w, b = _params(2, heads, d)
        y = _like(x, 7.0)
        mean, rstd = (torch.full((B, H, N), 7.0, device="cuda") for _ in range(2))
        sv.sv_layernorm(x, sv.desc_of(x), w, b, heads, 1e-5, y, sv.desc_of(y), mean, rstd)
        torch.cuda.synchronize()
        ref, rm, rr = orc.norm(to_host(x), to_host(w), to_host(b), 1e-5)
        assert np.abs(to_host(mean) - rm).max() <= 64 * E * 6 and np.abs(to_host(rstd) / rr - 1).max() <= 1000 * E
        assert np.abs(to_host(y) - ref).max() <= 1000 * E * 16
