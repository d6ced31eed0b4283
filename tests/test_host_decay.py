"""What the decayed linear attention's entry points refuse, before any launch; and how a call is cut into segments (csrc/decay_plan.hpp)."""
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


def _prompt(qkv=None, o=None, scale=1.0, wb=BIG, **at):
    p = dict(Q=A[0], K=A[1], V=A[2], g=A[3], lengths=None, s_in=A[4], s_out=A[5], O=A[6], ws=A[7])
    p.update(at)
    return _status(sv.sv_decay_linattn, p["Q"], p["K"], p["V"], qkv or _desc(), p["g"], p["lengths"], scale, p["s_in"], p["s_out"], p["O"],
                   o or _desc(), p["ws"], workspace_bytes=wb)


def _backward(qkv=None, o=None, scale=1.0, wb=BIG, **at):
    p = dict(Q=A[0], K=A[1], V=A[2], dO=A[3], g=A[4], lengths=None, s_in=A[5], ds_out=A[6], dQ=A[7], dK=A[8], dV=A[9], ds_in=A[10], ws=A[11])
    p.update(at)
    return _status(sv.sv_decay_linattn_backward, p["Q"], p["K"], p["V"], qkv or _desc(), p["dO"], o or _desc(), p["g"], p["lengths"], scale,
                   p["s_in"], p["ds_out"], p["dQ"], p["dK"], p["dV"], p["ds_in"], p["ws"], workspace_bytes=wb)


def _one(**kw):
    return _desc(**{**dict(N=1, stride_b=2 * 64, stride_h=64, stride_n=64), **kw})


def _token(qkv=None, o=None, scale=1.0, n_slots=4, **at):
    p = dict(Q=A[0], K=A[1], V=A[2], g=A[3], slots=A[4], s_in=A[5], s_out=A[5], O=A[6])
    p.update(at)
    return _status(sv.sv_decay_linattn_token, p["Q"], p["K"], p["V"], qkv or _one(), p["g"], p["slots"], n_slots, scale, p["s_in"], p["s_out"],
                   p["O"], o or _one())


@pytest.mark.parametrize("call,needed", [(_prompt, "Q K V g O ws"), (_backward, "Q K V dO g dQ dK dV ws"), (_token, "Q K V g s_in s_out O")])
def test_null_and_alignment(call, needed):
    for name in needed.split():
        assert call(**{name: None}) == 1, name
        if name != "g":
            assert call(**{name: A[15] + 8}) == 4, name


@pytest.mark.parametrize("call,base", [(_prompt, _desc), (_backward, _desc), (_token, _one)])
def test_descriptors(call, base):
    for kw, status in ((dict(d=48), 3), (dict(dtype=2), 3), (dict(B=0), 2), (dict(H=0), 2), (dict(N=0), 2), (dict(stride_n=32), 2),
                       (dict(stride_n=68), 4), (dict(stride_h=60), 4), (dict(H=1 << 25), 2)):
        assert call(qkv=base(**kw)) == status, kw
        assert call(o=base(**kw)) in (status, 2), kw
    assert call(o=base(B=2, stride_b=4 * 128 * 64)) == 2 and call(o=base(dtype=sv.SV_F32)) == 2          # not the inputs' shape or type
    assert call(o=base(d=32)) == 2
    for scale in (float("nan"), float("inf"), float("-inf")):
        assert call(scale=scale) == 5


@pytest.mark.parametrize("call,name", [(_prompt, "g"), (_prompt, "lengths"), (_backward, "g"), (_backward, "lengths"), (_token, "g"), (_token, "slots")])
def test_alignment_of_numbers(call, name):
    assert call(**{name: A[15] + 2}) == 4


def test_lanes_of_a_launch():
    """A launch has fewer than 2^32 lanes; larger calls are refused."""
    many = dict(B=1 << 12, H=1 << 12, N=1, d=128, stride_b=(1 << 12) * 128, stride_h=128, stride_n=128)
    assert _token(qkv=_desc(**many), o=_desc(**many)) == 2
    assert _prompt(qkv=_desc(**many), o=_desc(**many), s_in=None, s_out=None) == 2
    many.update(B=1 << 11)
    assert _backward(qkv=_desc(**many), o=_desc(**many), s_in=None, ds_out=None, ds_in=None) == 2


def test_far_rows():
    """64 rows span less than 2 GiB, or the call is refused: in-chunk offsets are 32-bit."""
    far = (1 << 31) // (64 * 2)
    for call in (_prompt, _backward):
        assert call(qkv=_desc(H=1, stride_n=far), o=_desc(H=1)) == 3
        assert call(qkv=_desc(H=1, stride_n=far - 8), o=_desc(H=1), wb=0) == 6           # gets as far as the workspace
        assert call(qkv=_desc(H=1, dtype=sv.SV_F32, stride_n=far // 2), o=_desc(H=1, dtype=sv.SV_F32)) == 3


def test_aliases():
    state = 2 * 64 * 64 * 4
    for name in ("Q", "K", "V"):
        assert _prompt(**{name: A[6]}) == 2
        assert _backward(**{name: A[7]}) == 2 and _backward(**{name: A[8]}) == 2 and _backward(**{name: A[9]}) == 2
        assert _token(**{name: A[6]}) == 2
    assert _prompt(s_out=A[4] + state - 16) == 2 and _prompt(s_out=A[4] - state + 16) == 2
    assert _prompt(s_out=A[4], wb=0) == 6 and _prompt(s_out=A[4] + state, wb=0) == 6          # in place, or side by side
    assert _backward(dQ=A[8]) == 2 and _backward(dV=A[8]) == 2
    assert _backward(ds_in=A[6]) == 2 and _backward(ds_in=A[5]) == 2 and _backward(ds_in=None, wb=0) == 6
    assert _token(s_out=A[5] + 4 * state - 16) == 2


def test_workspace_and_pool():
    for (B, H, N, d) in ((1, 2, 128, 64), (3, 20, 4000, 112), (1, 1, 1, 32), (2, 300, 100000, 128)):
        n, m = sv.sv_decay_linattn_workspace_bytes(B, H, N, d), sv.sv_decay_linattn_backward_workspace_bytes(B, H, N, d)
        assert n >= B * H * d * d * 4 and m >= 2 * B * H * d * d * 4 and n % 16 == 0 and m % 16 == 0
        dsc = _desc(B=B, H=H, N=N, d=d, stride_b=H * N * d, stride_h=N * d, stride_n=d)
        assert _prompt(qkv=dsc, o=dsc, wb=n - 1, s_in=None, s_out=None) == 6
        assert _backward(qkv=dsc, o=dsc, wb=m - 1, s_in=None, ds_out=None, ds_in=None) == 6
    for f in (sv.sv_decay_linattn_workspace_bytes, sv.sv_decay_linattn_backward_workspace_bytes):
        for d in (64, 128):                                                    # what a large call needs does for every smaller one
            sizes = [f(1, 20, n, d) for n in range(1, 6000, 61)] + [f(1, 20, 1 << 22, d)]
            assert sizes == sorted(sizes)
            sizes = [f(b, 3, 1000, d) for b in range(1, 400, 7)] + [f(b, 8, 1000, d) for b in (150, 151)]
            assert sizes == sorted(sizes)
    for bad in ((0, 2, 128, 64), (1, 0, 128, 64), (1, 2, 0, 64), (1, 2, 128, 48), (1 << 12, 1 << 13, 128, 64)):
        assert sv.sv_decay_linattn_workspace_bytes(*bad) == 0 and sv.sv_decay_linattn_backward_workspace_bytes(*bad) == 0
    assert _token(qkv=_one(N=2, stride_n=128), o=_one(N=2, stride_n=128)) == 2
    assert _token(n_slots=0) == 2 and _token(n_slots=-1) == 2
    assert _token(qkv=_one(B=5), o=_one(B=5), slots=None) == 2                 # five rows, four states


def test_plan(tmp_path):
    exe = tmp_path / "host_decay_plan"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", os.path.join(ROOT, "tests", "host_decay_plan.cpp"), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0 and res.stdout.startswith("OK"), res.stdout
