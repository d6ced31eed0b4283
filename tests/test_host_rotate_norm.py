"""What the rotation and the layer norm refuse, before any launch; and the forms that rows of every width get (csrc/norm_plan.hpp)."""
import os
import subprocess

import pytest

import paper_2509_24695_amd as sv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [0x100000 * (i + 1) for i in range(20)]          # aligned, never dereferenced: every call below fails before a launch
BIG = 1 << 40


def _desc(**kw):
    return sv.TensorDesc(**{**dict(B=1, H=2, N=128, d=64, stride_b=2 * 128 * 64, stride_h=128 * 64, stride_n=64, dtype=sv.SV_BF16), **kw})


def _status(f, *a, **kw):
    with pytest.raises(sv.SvError) as e:
        f(*a, **kw)
    return e.value.status


def _rope(**kw):
    return sv.Rope3D(**{**dict(frames=2, rows=8, cols=8, n_t=12, n_h=10, n_w=10, cs_t=A[10], cs_h=A[11], cs_w=A[12]), **kw})


def _rotate(x=None, y=None, rope=None, **at):
    p = dict(Q=A[0], K=A[1], positions=None, YQ=A[2], YK=A[3])
    p.update(at)
    return _status(sv.sv_rope3d_rotate, p["Q"], p["K"], x or _desc(), rope or _rope(), p["positions"], 0, p["YQ"], p["YK"], y or _desc())


def test_rotate_refusals():
    for name in ("Q", "YQ", "K", "YK"):
        assert _rotate(**{name: None}) == 1, name                     # K and YK come together
        assert _rotate(**{name: A[9] + 8}) == 4, name
    assert _status(sv.sv_rope3d_rotate, A[0], None, _desc(), None, None, 0, A[2], None, _desc()) == 1
    assert _status(sv.sv_rope3d_rotate, A[0], None, None, _rope(), None, 0, A[2], None, _desc()) == 1
    assert _rotate(positions=A[8] + 2) == 4
    for kw, status in ((dict(d=48), 3), (dict(dtype=7), 3), (dict(N=0), 2), (dict(stride_n=60), 2), (dict(stride_n=68), 4), (dict(B=2), 2)):
        assert _rotate(x=_desc(**kw)) == status, kw
        assert _rotate(y=_desc(**kw)) in (status, 2), kw
    assert _rotate(y=_desc(dtype=sv.SV_F32)) == 2 and _rotate(y=_desc(d=32)) == 2
    for kw in (dict(frames=0), dict(rows=-1), dict(cols=9), dict(frames=3), dict(n_t=-1, n_w=23), dict(n_t=13), dict(n_w=9),
               dict(frames=1 << 20, rows=1 << 20, cols=1 << 24)):
        assert _rotate(rope=_rope(**kw)) == 2, kw
    for kw in (dict(cs_t=None), dict(cs_h=None), dict(cs_w=None)):
        assert _rotate(rope=_rope(**kw)) == 1, kw
    for kw in (dict(cs_t=A[10] + 4), dict(cs_h=A[10] + 4), dict(cs_w=A[10] + 4)):
        assert _rotate(rope=_rope(**kw)) == 4, kw
    apart = _desc(stride_h=130 * 64, stride_b=2 * 130 * 64)
    assert _rotate(YQ=A[0], y=apart) == 2 and _rotate(YK=A[1], y=apart) == 2          # in place with other strides
    assert _rotate(YQ=A[1]) == 2 and _rotate(YK=A[0]) == 2 and _rotate(YQ=A[3]) == 2


def test_lanes_of_a_launch():
    """A launch has fewer than 2^32 lanes; larger calls are refused."""
    n = 1 << 28                                                       # 16 tokens a workgroup of 256
    long = _desc(H=1, N=n, d=128, stride_n=128, stride_h=n * 128, stride_b=n * 128)
    assert _rotate(x=long, y=long, rope=_rope(frames=1 << 8, rows=1 << 10, cols=1 << 10, n_t=24, n_h=20, n_w=20)) == 2
    heads = _desc(H=1 << 24, N=1, d=8, stride_n=8, stride_h=8, stride_b=8 << 24)
    assert _norm(x=heads, y=heads, heads=1 << 24) == 2
    assert _norm_backward(x=heads, dy=heads, dx=heads, heads=1 << 24) == 2
    wide = _desc(H=1 << 16, N=1, d=8192, stride_n=8192, stride_h=8192, stride_b=8192 << 16)     # 256 workgroups a head add the partial sums up
    assert _norm_backward(x=wide, dy=wide, dx=wide, heads=1 << 16) == 2


def _norm(x=None, y=None, heads=1, eps=1e-5, **at):
    p = dict(X=A[0], w=A[1], b=A[2], Y=A[3], mean=A[4], rstd=A[5])
    p.update(at)
    return _status(sv.sv_layernorm, p["X"], x or _desc(), p["w"], p["b"], heads, eps, p["Y"], y or _desc(), p["mean"], p["rstd"])


def _norm_backward(x=None, dy=None, dx=None, heads=1, wb=BIG, **at):
    p = dict(X=A[0], dY=A[1], w=A[2], mean=A[3], rstd=A[4], dX=A[5], dw=A[6], db=A[7], ws=A[8])
    p.update(at)
    return _status(sv.sv_layernorm_backward, p["X"], x or _desc(), p["dY"], dy or _desc(), p["w"], heads, p["mean"], p["rstd"], p["dX"], dx or _desc(),
                   p["dw"], p["db"], p["ws"], workspace_bytes=wb)


def _row(d, **kw):
    return _desc(d=d, stride_n=d, stride_h=128 * d, stride_b=2 * 128 * d, **kw)


def test_norm_refusals():
    for name in ("X", "Y", "mean", "rstd"):
        assert _norm(**{name: None}) == 1, name
    for name in ("X", "Y", "w", "b", "mean", "rstd"):
        assert _norm(**{name: A[9] + 8}) == 4, name
    for d, dtype, status in ((12, sv.SV_BF16, 4), (8200, sv.SV_BF16, 3), (8196, sv.SV_F32, 3), (64, 4, 3)):
        assert _norm(x=_row(d, dtype=dtype)) == status, (d, dtype)
        assert _norm_backward(x=_row(d, dtype=dtype)) == status, (d, dtype)
    odd = _desc(d=12, stride_n=16, stride_h=128 * 16, stride_b=2 * 128 * 16)
    assert _norm(x=odd) == 3 and _norm_backward(x=odd) == 3                             # 12 features of bf16 are no whole pieces
    assert _norm(x=_desc(d=0)) == 3 and _norm(x=_desc(d=-8)) == 3
    assert _norm(y=_desc(N=64)) == 2 and _norm(y=_row(64, dtype=sv.SV_F32)) == 2 and _norm(y=_row(72)) == 2
    for heads in (0, -1, 3):
        assert _norm(heads=heads) == 2 and _norm_backward(heads=heads) == 2
    for eps in (-1e-9, float("nan"), float("inf")):
        assert _norm(eps=eps) == 5
    assert _norm(Y=A[0], y=_desc(stride_h=130 * 64, stride_b=2 * 130 * 64)) == 2 and _norm(mean=A[5]) == 2
    huge = dict(B=1 << 8, H=1 << 16, N=128, stride_b=1 << 40, stride_h=1 << 14, stride_n=64)
    assert _norm(x=_desc(**huge)) == 2 and _norm_backward(x=_desc(**huge)) == 2       # 2^31 rows


def test_norm_backward_refusals():
    for name in ("X", "dY", "mean", "rstd", "dX", "ws"):
        assert _norm_backward(**{name: None}) == 1, name
    for name in ("X", "dY", "w", "mean", "rstd", "dX", "dw", "db", "ws"):
        assert _norm_backward(**{name: A[9] + 8}) == 4, name
    assert _norm_backward(dy=_desc(N=64)) == 2 and _norm_backward(dx=_row(72)) == 2
    assert _norm_backward(dX=A[0]) == 2 and _norm_backward(dX=A[1], dx=_desc(stride_h=130 * 64, stride_b=2 * 130 * 64)) == 2
    assert _norm_backward(dw=A[7]) == 2 and _norm_backward(dw=A[2]) == 2 and _norm_backward(db=A[2]) == 2
    need = sv.sv_layernorm_backward_workspace_bytes(1, 2, 128, 64)
    assert need > 0 and need % 16 == 0
    assert _norm_backward(wb=1000) == 6
    for bad in ((0, 1, 1, 64), (1, 0, 1, 64), (1, 1, 0, 64), (1, 1, 1, 0), (1, 1, 1, 66), (1, 1, 1, 8196), (1 << 12, 1 << 13, 1, 64)):
        assert sv.sv_layernorm_backward_workspace_bytes(*bad) == 0
    assert sv.sv_layernorm_backward_workspace_bytes(1, 3000, 7, 64) >= 3000 * 2 * 64 * 4          # a partial sum of each head at least


def test_norm_plan(tmp_path):
    exe = tmp_path / "host_norm_plan"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", os.path.join(ROOT, "tests", "host_norm_plan.cpp"), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0 and res.stdout.startswith("OK"), res.stdout
