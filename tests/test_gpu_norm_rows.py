"""Layer norm over more rows than its workgroups take at once, for every form in which a row lies in several waves: sums across waves one after the
other, the next row on its way meanwhile, in place too.  Rows leave some lanes without one at the end.  Bounds as in test_gpu_norm.py; the
reference is worked out in 64 bits on the device.

test_host_norm_cases.py holds the cases to what they are here for."""
import pytest

import paper_2509_24695_amd as sv
from tests.gpu_util import say
from tests.test_gpu_norm import E, U, _params, _rows, _space, _torch

pytestmark = pytest.mark.gpu

# d, dtype, rows, backward
FORWARD = [(3080, "bf16", 4101), (4096, "bf16", 8195), (4104, "bf16", 2051), (6144, "bf16", 4099), (6152, "bf16", 2051), (8192, "bf16", 4097),
           (1540, "f32", 4101), (2052, "f32", 2051), (3064, "f32", 4097), (4096, "f32", 2049), (4100, "f32", 2051), (8192, "f32", 4097)]
BACKWARD = [(1544, "bf16", 1027), (2048, "bf16", 2051), (2240, "bf16", 1029), (4088, "bf16", 1027), (4104, "bf16", 259), (6144, "bf16", 515),
            (6152, "bf16", 259), (8192, "bf16", 515), (772, "f32", 1027), (1284, "f32", 1027), (1540, "f32", 1029), (2052, "f32", 515), (3064, "f32", 1027),
            (4096, "f32", 259), (4100, "f32", 259), (8192, "f32", 515)]


def _id(c):
    return f"{c[2]}x{c[0]}-{c[1]}"


@pytest.mark.parametrize("case", FORWARD, ids=_id)
def test_forward(case):
    torch = _torch()
    d, dtype, N = case
    say(f"norm rows forward {_id(case)}")
    x = _rows(31, 1, 1, N, d, dtype, "bhnd", 0.5)
    w, b = _params(32, 1, d)
    y, mean, rstd = torch.full_like(x, 7.0), torch.full((1, 1, N), 7.0, device="cuda"), torch.full((1, 1, N), 7.0, device="cuda")
    sv.sv_layernorm(x, sv.desc_of(x), w, b, 1, 1e-5, y, sv.desc_of(y), mean, rstd)
    torch.cuda.synchronize()
    xd, wd, bd = x.double(), w.double()[None, None], b.double()[None, None]
    rm = xd.mean(-1)
    off = xd - rm[..., None]
    rr = (off.square().mean(-1) + 1e-5).rsqrt()
    A = xd.abs().mean(-1)
    part = (xd.abs() + A[..., None]) * rr[..., None]
    S = part.square().mean(-1).sqrt()
    assert bool(((mean.double() - rm).abs() <= 64 * E * A).all()) and bool(((rstd.double() - rr).abs() <= (64 + 65 * S) * E * rr).all())
    normed = off * rr[..., None]
    ref = normed * wd + bd
    tol = ((U if dtype == "bf16" else E) + 2 * E) * ref.abs() + (130 + 65 * S[..., None]) * E * wd.abs() * (normed.abs() + part)
    assert bool(((y.double() - ref).abs() <= tol).all())
    sv.sv_layernorm(x, sv.desc_of(x), w, b, 1, 1e-5, x, sv.desc_of(x), None, None)
    torch.cuda.synchronize()
    assert torch.equal(x, y)


@pytest.mark.parametrize("case", BACKWARD, ids=_id)
def test_backward(case):
    torch = _torch()
    d, dtype, N = case
    say(f"norm rows backward {_id(case)}")
    x, dy = _rows(33, 1, 1, N, d, dtype, "bhnd", 0.5), _rows(34, 1, 1, N, d, dtype, "bhnd", 0.1)
    w, _ = _params(35, 1, d)
    xd, g, wd = x.double(), dy.double(), w.double()[None, None]
    mean = xd.mean(-1).float()
    rstd = ((xd - xd.mean(-1, keepdim=True)).square().mean(-1) + 1e-5).rsqrt().float()
    dx, dw, db, ws = torch.full_like(x, 7.0), torch.full((1, d), 7.0, device="cuda"), torch.full((1, d), 7.0, device="cuda"), _space(1, 1, N, d)
    sv.sv_layernorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, 1, mean, rstd, dx, sv.desc_of(dx), dw, db, ws)
    torch.cuda.synchronize()
    m, r = mean.double()[..., None], rstd.double()[..., None]
    xh, t = (xd - m) * r, wd * g
    size = (xd.abs() + m.abs()) * r
    along = (t * xh).mean(-1, keepdim=True)
    ref = r * (t - t.mean(-1, keepdim=True) - xh * along)
    mag = r * (t.abs() + t.abs().mean(-1, keepdim=True) + (xh.abs() + size) * (t * xh).abs().mean(-1, keepdim=True)
               + xh.abs() * (t.abs() * size).mean(-1, keepdim=True))
    assert bool(((dx.double() - ref).abs() <= (U if dtype == "bf16" else E) * ref.abs() + 80 * E * mag).all())
    c = N / 32 + 80
    assert bool(((dw.double() - (g * xh).sum(2)[0]).abs() <= c * E * (g.abs() * (xh.abs() + size)).sum(2)[0]).all())
    assert bool(((db.double() - g.sum(2)[0]).abs() <= c * E * g.abs().sum(2)[0]).all())
    dw2, db2 = torch.full_like(dw, 7.0), torch.full_like(db, 7.0)
    sv.sv_layernorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, 1, mean, rstd, dy, sv.desc_of(dy), dw2, db2, ws)      # dx over dy
    torch.cuda.synchronize()
    assert torch.equal(dy, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)
