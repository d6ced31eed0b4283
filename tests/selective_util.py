"""Helpers of the GPU tests of the short convolution, the selective scan and the group norm: tensors in every layout, and comparison with a
bound for each element."""
from __future__ import annotations

import numpy as np

import paper_2509_24695_amd as sv
from tests.gpu_util import to_host

E = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": E}           # one rounding, relative


def _torch():
    import torch
    return torch


def dtype_of(dtype):
    torch = _torch()
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def place(x, layout):
    """A CPU tensor [B][H][N][d] on the device: heads outside tokens ("bhnd"), token-major ("bnhd"), or with rows apart inside a larger tensor
    of NaN ("apart")."""
    torch = _torch()
    if layout == "bhnd":
        return x.contiguous().cuda()
    if layout == "bnhd":
        return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
    B, H, N, d = x.shape
    wide = torch.full((B, N + 3, H, d + 32), float("nan"), dtype=x.dtype, device="cuda")
    view = wide[:, 1:N + 1, :, 16:16 + d].permute(0, 2, 1, 3)
    view.copy_(x)
    return view


def draw(seed, shape, dtype, layout="bhnd", scale=1.0, shift=0.0):
    torch = _torch()
    x = scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed)) + shift
    return place(x.to(dtype_of(dtype)), layout)


def floats(seed, *shape, scale=1.0):
    torch = _torch()
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).cuda()


def like(x, value=float("nan")):
    """A tensor that lies as x does, and what surrounds it, all of one value."""
    torch = _torch()
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device).fill_(value)


def f64(x):
    return None if x is None else to_host(x).astype(np.float64)


def space(nbytes):
    assert nbytes > 0
    return _torch().empty(nbytes, dtype=_torch().uint8, device="cuda").fill_(255)


def ints(v):
    return None if v is None else _torch().tensor(v, dtype=_torch().int32, device="cuda")


def spoil(x, lengths):
    """Rows behind the last token of each sequence become NaN."""
    for b, n in enumerate(lengths or []):
        x[b, :, n:] = float("nan")


def check(name, got, want, bound, dtype):
    """|got - want| <= bound e + one rounding to dtype (and the smallest normal numbers of fp32); where `want` is NaN nothing was written:
    `got` still holds the NaN it was filled with."""
    g = f64(got)
    assert g.shape == want.shape, (name, g.shape, want.shape)
    hole = np.isnan(want)
    assert np.isnan(g[hole]).all(), f"{name}: rows behind the last token were written"
    off = np.abs(g - want)[~hole]
    allowed = (bound * E + U[dtype] * (np.abs(want) + bound * E) + 2.0 ** -125)[~hole]
    bad = ~(off <= allowed)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.where(bad, off / allowed, 0)):.3g} of the bound, first {np.argwhere(~hole)[np.argmax(bad)]}"


def same_bits(a, b):
    torch = _torch()
    assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def replayed(call, change, outputs, times=3):
    """Captures `call`, replays it with inputs that `change(i)` rewrites, and compares every replay with the eager result."""
    torch = _torch()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(torch.cuda.current_stream())
    for i in range(times):
        change(i)
        for o in outputs:
            o.fill_(float("nan"))
        call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        eager = [o.clone() for o in outputs]
        for o in outputs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for o, e in zip(outputs, eager):
            same_bits(o, e)
