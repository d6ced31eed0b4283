"""What the short convolution refuses, before any launch."""
import pytest

import paper_2509_24695_amd as sv
from paper_2509_24695_amd import binding

A = [0x1000000 * (i + 1) for i in range(20)]         # aligned, never dereferenced: every call below fails before a launch
BIG = 1 << 40


@pytest.fixture(params=["module", "ctypes"], autouse=True)
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
    p = dict(X=A[0], x=_desc(), W=A[1], b=A[2], taps=4, silu=True, lengths=None, ci=A[3], co=A[4], Y=None, y=_desc())
    p.update(kw)
    return _status(sv.sv_causal_conv, *p.values())


def _token(**kw):
    one = _desc(N=1)
    p = dict(X=A[0], x=one, W=A[1], b=A[2], taps=4, silu=1, slots=A[5], n=7, ci=A[3], co=A[4], Y=None, y=one)
    p.update(kw)
    return _status(sv.sv_causal_conv_token, *p.values())


def _backward(**kw):
    p = dict(X=A[0], x=_desc(), dY=A[1], dy=_desc(), W=A[2], b=A[3], taps=4, silu=1, lengths=None, ci=A[4], dco=A[5], dX=None, dx=_desc(), dci=A[6], dW=A[7],
             db=A[8], ws=A[9], wb=BIG)
    p.update(kw)
    return _status(sv.sv_causal_conv_backward, *p.values())


DESCS = ((dict(d=60), 4), (dict(d=0), 3), (dict(d=8200, H=1, stride_n=8200), 3), (dict(dtype=7), 3), (dict(N=0), 2), (dict(B=0), 2), (dict(stride_n=56), 2), (dict(stride_n=68), 4),
         (dict(B=2), 0), (dict(stride_h=64), 2))


def test_forward():
    assert _forward() == 1                                            # no Y
    for name in ("X", "W"):
        assert _forward(Y=A[9], **{name: None}) == 1
    for name in ("X", "W", "b", "ci", "co", "Y"):
        assert _forward(**{"Y": A[9], name: A[10] + 8}) == 4, name
    assert _forward(Y=A[9], lengths=A[11] + 2) == 4
    assert _forward(Y=A[9], x=None) == 1 and _forward(Y=A[9], y=None) == 1
    for kw, status in DESCS:
        if status in (2, 3):
            assert _forward(Y=A[9], x=_desc(**kw)) == status, kw
            assert _forward(Y=A[9], y=_desc(**kw)) == status, kw
    assert _forward(Y=A[9], x=_desc(stride_n=68)) == 4
    for kw in (dict(dtype=sv.SV_F32), dict(d=32), dict(N=64), dict(H=1)):
        assert _forward(Y=A[9], y=_desc(**kw)) == 2, kw
    for taps in (1, 5, 0, -4):
        assert _forward(Y=A[9], taps=taps) == 3
    for act in (2, -1):
        assert _forward(Y=A[9], silu=act) == 5
    assert _forward(Y=A[0]) == 2                                      # in place
    assert _forward(Y=A[9], co=A[3] + 16) == 2 and _forward(Y=A[9], co=A[9]) == 2 and _forward(Y=A[9], co=A[0]) == 2
    n = (1 << 31) - 1                                                 # tokens are counted a little past the last
    assert _forward(Y=A[9], **{k: _desc(H=1, N=n, d=8, stride_n=8, stride_h=8 * n, stride_b=8 * n) for k in ("x", "y")}) == 2
    assert _forward(Y=A[9], **{k: _desc(H=1, N=n, d=2048, stride_n=2048, stride_h=n * 2048, stride_b=n * 2048) for k in ("x", "y")}) == 2
    assert _forward(Y=A[9], **{k: _desc(H=1 << 20, N=1, d=4096, stride_n=4096, stride_h=4096, stride_b=1 << 40) for k in ("x", "y")}) == 2


def test_token():
    assert _token() == 1
    for name in ("X", "W", "ci", "co"):
        assert _token(Y=A[9], **{name: None}) == 1, name
    for name in ("X", "W", "b", "ci", "co", "Y"):
        assert _token(**{"Y": A[9], name: A[10] + 8}) == 4, name
    assert _token(Y=A[9], slots=A[5] + 1) == 4
    assert _token(Y=A[9], x=_desc(), y=_desc()) == 2                  # more than one token
    assert _token(Y=A[9], n=0) == 2 and _token(Y=A[9], n=-1) == 2
    two = _desc(N=1, B=9, stride_b=1 << 20)
    assert _token(Y=A[9], x=two, y=two, slots=None, n=8) == 2
    assert _token(Y=A[0]) == 2 and _token(Y=A[9], co=A[3] + 16) == 2 and _token(Y=A[9], taps=5) == 3 and _token(Y=A[9], silu=2) == 5


def test_backward():
    assert _backward() == 1
    for name in ("X", "dY", "W", "ws"):
        assert _backward(dX=A[10], **{name: None}) == 1, name
    for name in ("X", "dY", "W", "b", "ci", "dco", "dX", "dci", "dW", "db", "ws"):
        assert _backward(**{"dX": A[10], name: A[11] + 8}) == 4, name
    for name in ("x", "dy", "dx"):
        assert _backward(dX=A[10], **{name: None}) == 1
        assert _backward(dX=A[10], **{name: _desc(N=64)}) == 2
        assert _backward(dX=A[10], **{name: _desc(d=60, stride_n=64)}) in (2, 3)
    assert _backward(dX=A[10], lengths=A[12] + 2) == 4
    assert _backward(dX=A[10], taps=5) == 3 and _backward(dX=A[10], silu=-1) == 5
    assert _backward(dX=A[0]) == 2 and _backward(dX=A[1]) == 2
    assert _backward(dX=A[10], dci=A[5]) == 2 and _backward(dX=A[10], dci=A[4]) == 2 and _backward(dX=A[10], dci=A[10]) == 2
    assert _backward(dX=A[10], dW=A[8]) == 2 and _backward(dX=A[10], dW=A[2]) == 2 and _backward(dX=A[10], db=A[3]) == 2
    assert _backward(dX=A[10], wb=64) == 6


def test_workspace():
    f = sv.sv_causal_conv_backward_workspace_bytes
    for bad in ((0, 1, 1, 8), (1, 0, 1, 8), (1, 1, 0, 8), (1, 1, 1, 0), (1, 1, 1, 6), (1, 1, 1, 8196), (1 << 13, 1 << 12, 1, 8)):
        assert f(*bad) == 0
    assert 0 < f(1, 1, 1, 8) <= 1 << 12
    last = 0
    for n in (1, 31, 32, 33, 500, 513, 4680, 32760, 75600, 1 << 20):   # never less for more
        assert f(2, 20, n, 112) >= last
        last = f(2, 20, n, 112)
        assert f(3, 20, n, 112) >= last and f(2, 21, n, 112) >= last
