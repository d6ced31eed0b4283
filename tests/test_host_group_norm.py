"""What the group norm refuses, before any launch, and how its calls are cut up (csrc/group_plan.hpp)."""
import os
import subprocess

import pytest

import paper_2509_24695_amd as sv
from paper_2509_24695_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [0x1000000 * (i + 1) for i in range(40)]         # aligned, never dereferenced: every call below fails before a launch
BIG = 1 << 40


@pytest.fixture(params=["module", "ctypes"])
def route(request, monkeypatch):
    lib = sv.load_library()
    monkeypatch.setattr(binding, "_entry", binding._load_entry(lib) if request.param == "module" else binding._CtypesCalls(lib))


def _desc(**kw):
    return sv.TensorDesc(**{**dict(B=1, H=2, N=128, d=64, stride_b=2 * 128 * 64, stride_h=128 * 64, stride_n=64, dtype=sv.SV_BF16), **kw})


def _status(f, *a, **kw):
    with pytest.raises(sv.SvError) as e:
        f(*a, **kw)
    return e.value.status


def _forward(**kw):
    p = dict(X=A[0], x=_desc(), w=A[1], b=A[2], groups=4, eps=1e-5, silu=True, Y=None, y=_desc(), mean=A[3], rstd=A[4], ws=A[5], wb=BIG)
    p.update(kw)
    return _status(sv.sv_groupnorm, *p.values())


def _backward(**kw):
    p = dict(X=A[0], x=_desc(), dY=A[1], dy=_desc(), w=A[2], b=A[3], groups=4, silu=1, mean=A[4], rstd=A[5], dX=None, dx=_desc(), dw=A[6], db=A[7], ws=A[8], wb=BIG)
    p.update(kw)
    return _status(sv.sv_groupnorm_backward, *p.values())


DESCS = ((dict(d=60, stride_n=64), 3), (dict(d=8200, H=1, stride_n=8200), 3), (dict(dtype=7), 3), (dict(N=0), 2), (dict(B=0), 2), (dict(stride_n=56), 2), (dict(stride_n=68), 4),
         (dict(stride_h=64), 2), (dict(H=1, N=(1 << 31) - 1, stride_h=1 << 40, stride_b=1 << 40, B=2), 2))


def test_forward(route):
    assert _forward() == 1
    given = dict(Y=A[30])
    for name in ("X", "ws", "x", "y", "mean", "rstd"):                # statistics come together
        assert _forward(**{**given, name: None}) == 1, name
    for name in ("X", "w", "b", "Y", "mean", "rstd", "ws"):
        assert _forward(**{**given, name: A[31] + 8}) == 4, name
    for kw, status in DESCS:
        assert _forward(Y=A[30], x=_desc(**kw)) == status, kw
        assert _forward(Y=A[30], y=_desc(**kw)) == status, kw
    for kw in (dict(dtype=sv.SV_F32), dict(d=32), dict(N=64), dict(H=1)):
        assert _forward(Y=A[30], y=_desc(**kw)) == 2, kw
    for groups in (0, -4, 5, 128):
        assert _forward(Y=A[30], groups=groups) == 2
    for eps in (-1e-9, float("nan"), float("inf")):
        assert _forward(Y=A[30], eps=eps) == 5
    assert _forward(Y=A[30], silu=2) == 5 and _forward(Y=A[30], silu=-1) == 5
    assert _forward(Y=A[0], y=_desc(stride_h=130 * 64, stride_b=260 * 64)) == 2       # in place with other strides
    assert _forward(Y=A[30], mean=A[4]) == 2 and _forward(Y=A[30], wb=64) == 6


def test_backward(route):
    assert _backward() == 1
    given = dict(dX=A[30])
    for name in ("X", "dY", "mean", "rstd", "ws", "x", "dy", "dx"):
        assert _backward(**{**given, name: None}) == 1, name
    for name in ("X", "dY", "w", "b", "mean", "rstd", "dX", "dw", "db", "ws"):
        assert _backward(**{**given, name: A[31] + 8}) == 4, name
    for name in ("x", "dy", "dx"):
        for kw, status in DESCS:
            assert _backward(**{**given, name: _desc(**kw)}) == status, kw
    for kw in (dict(dtype=sv.SV_F32), dict(d=32), dict(N=64), dict(H=1)):
        assert _backward(dX=A[30], dy=_desc(**kw)) == 2 and _backward(dX=A[30], dx=_desc(**kw)) == 2, kw
    assert _backward(dX=A[30], groups=7) == 2 and _backward(dX=A[30], silu=2) == 5
    assert _backward(dX=A[0]) == 2 and _backward(dX=A[1], dx=_desc(stride_h=130 * 64, stride_b=260 * 64)) == 2
    assert _backward(dX=A[30], dw=A[7]) == 2 and _backward(dX=A[30], dw=A[2]) == 2 and _backward(dX=A[30], db=A[3]) == 2
    assert _backward(dX=A[30], wb=64) == 6


def test_workspaces():
    f, g = sv.sv_groupnorm_workspace_bytes, sv.sv_groupnorm_backward_workspace_bytes
    for bad in ((0, 1, 1, 8, 1), (1, 0, 1, 8, 1), (1, 1, 0, 8, 1), (1, 1, 1, 0, 1), (1, 1, 1, 6, 1), (1, 1, 1, 8196, 1), (1, 1, 1, 8, 3), (1, 1, 1, 8, 0), (1 << 13, 1 << 12, 1, 8, 1)):
        assert f(*bad) == 0 and g(*bad) == 0
    for B, H, d, G in ((1, 1, 2240, 32), (2, 21, 320, 32), (7, 300, 32, 1)):
        last = 0, 0
        for N in (1, 31, 33, 64, 500, 1560, 32760, 75600):             # never less for more rows, batches or heads
            now = f(B, H, N, d, G), g(B, H, N, d, G)
            assert now[0] >= last[0] and now[1] >= last[1]
            for b, h in ((B + 1, H), (B, H + 1)):
                assert f(b, h, N, d, G) >= now[0] and g(b, h, N, d, G) >= now[1]
            last = now


def test_plans(tmp_path):
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", "host_row_plans.cpp"), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)
