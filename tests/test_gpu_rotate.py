"""The rotation on its own (sv_rope3d_rotate) against complex products in 64 bits.  Each output is x cos -+ y sin with at most two roundings
of 2^-24 of its terms, then one to the tensors' type (half a step: 2^-8 of bf16)."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
import sv_workloads as wl
from oracle import layer_oracle as orc
from tests.gpu_util import say, to_host

pytestmark = pytest.mark.gpu

U, E = 2.0 ** -8, 2.0 ** -24


def _torch():
    import torch
    return torch


def _draw(seed, B, H, N, d, dtype, layout, count):
    torch = _torch()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(seed)
    if layout == "packed":
        x = torch.randn((B, N, count, H, d), generator=gen).to(dt).cuda()
        return [x[:, :, i].permute(0, 2, 1, 3) for i in range(count)]
    shape = (B, H, N, d) if layout == "bhnd" else (B, N, H, d)
    xs = [torch.randn(shape, generator=gen).to(dt).cuda() for _ in range(count)]
    return xs if layout == "bhnd" else [x.permute(0, 2, 1, 3) for x in xs]


def _tables(grid, d, t0=0):
    return wl.rope_tables_3d_factored(*grid, d, t0=t0)


def _rope(tables):
    return sv.Rope3D.from_tensors(*(_torch().from_numpy(t).cuda() for t in tables))


def _check(got, x, tables, positions, inverse, dtype, kept, what):
    x = to_host(x).astype(np.float64)
    got = to_host(got)
    ref = orc.rotate(x, tables, positions, inverse, kept)
    size = np.abs(x[..., 0::2]) + np.abs(x[..., 1::2])
    tol = np.repeat(2 * E * size, 2, axis=-1) + (U if dtype == "bf16" else E) * np.abs(ref)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} beyond the bound"


CASES = [   # B, H, (frames, rows, cols), d, dtype, layout
    (1, 1, (1, 1, 1), 64, "bf16", "bhnd"),
    (2, 3, (1, 1, 7), 32, "f32", "bnhd"),
    (1, 20, (3, 5, 7), 112, "bf16", "packed"),
    (2, 5, (2, 9, 11), 112, "f32", "bnhd"),
    (3, 7, (5, 3, 13), 128, "bf16", "bhnd"),
    (1, 33, (2, 4, 8), 128, "f32", "packed"),
    (1, 9, (7, 10, 12), 64, "bf16", "bnhd"),
    (2, 2, (4, 6, 50), 32, "bf16", "bhnd"),
    (1, 3, (21, 30, 52), 64, "f32", "bhnd"),                 # all heads in one workgroup's loop
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}H{c[1]}-{'x'.join(map(str, c[2]))}-d{c[3]}-{c[4]}-{c[5]}")
@pytest.mark.parametrize("inverse", [0, 1])
def test_grid(case, inverse):
    torch = _torch()
    B, H, grid, d, dtype, layout = case
    N = int(np.prod(grid))
    say(f"rotate grid {case} inverse={inverse}")
    q, k = _draw(3, B, H, N, d, dtype, layout, 2)
    tables, positions = _tables(grid, d, t0=2), orc.grid_positions(*grid)
    r = _rope(tables)
    yq, yk = (torch.full((B, H, N, d), 7.0, dtype=q.dtype, device="cuda") for _ in range(2))
    sv.sv_rope3d_rotate(q, k, sv.desc_of(q), r, None, inverse, yq, yk, sv.desc_of(yq))
    torch.cuda.synchronize()
    _check(yq, q, tables, positions, inverse, dtype, None, "q")
    _check(yk, k, tables, positions, inverse, dtype, None, "k")
    # q alone, and in place
    alone = torch.full_like(yq, 7.0)
    sv.sv_rope3d_rotate(q, None, sv.desc_of(q), r, None, inverse, alone, None, sv.desc_of(alone))
    sv.sv_rope3d_rotate(q, k, sv.desc_of(q), r, None, inverse, q, k, sv.desc_of(q))
    torch.cuda.synchronize()
    assert torch.equal(alone, yq) and torch.equal(q, yq) and torch.equal(k, yk)


@pytest.mark.parametrize("B,H,N,d,dtype,layout", [(1, 4, 1, 64, "bf16", "packed"), (3, 5, 77, 112, "bf16", "packed"), (2, 16, 300, 128, "f32", "bhnd"),
                                                   (2, 3, 50, 32, "bf16", "bnhd")])
@pytest.mark.parametrize("inverse", [0, 1])
def test_positions(B, H, N, d, dtype, layout, inverse):
    """Any places in any order, more than once; tokens outside a table on either side keep their rows."""
    torch = _torch()
    grid = (5, 7, 9)
    say(f"rotate positions B={B} H={H} N={N} d={d} {dtype} inverse={inverse}")
    rng = np.random.default_rng(8)
    positions = np.stack([rng.integers(0, m, (B, N)) for m in grid], axis=-1).astype(np.int32)
    if N > 20:
        positions[0, 3:9] = [[-1, 0, 0], [5, 0, 0], [0, -7, 0], [0, 7, 0], [0, 0, -2 ** 31], [0, 0, 9]]
        positions[-1, N - 5:] = -1
        positions[:, 12] = positions[:, 13]
    q, k = _draw(5, B, H, N, d, dtype, layout, 2)
    tables = _tables(grid, d)
    yq, yk = (_torch().empty_strided(q.shape, q.stride(), dtype=q.dtype, device="cuda").fill_(7.0) for _ in range(2))
    sv.sv_rope3d_rotate(q, k, sv.desc_of(q), _rope(tables), torch.from_numpy(positions).cuda(), inverse, yq, yk, sv.desc_of(yq))
    torch.cuda.synchronize()
    kept = np.full(tuple(q.shape), 7.0)
    _check(yq, q, tables, positions, inverse, dtype, kept, "q")
    _check(yk, k, tables, positions, inverse, dtype, kept, "k")


def test_inverse_is_the_gradient():
    """<R x, g> = <x, R^T g> for every x and g: the rotation's backward pass is its inverse (fp32: N H d products off by 4 x 2^-24 of their size each)."""
    torch = _torch()
    B, H, grid, d = 2, 4, (2, 5, 6), 64
    N = int(np.prod(grid))
    x, = _draw(1, B, H, N, d, "f32", "bhnd", 1)
    g, = _draw(2, B, H, N, d, "f32", "bhnd", 1)
    r = _rope(_tables(grid, d))
    y, back = torch.empty_like(x), torch.empty_like(x)
    say("rotate inverse")
    sv.sv_rope3d_rotate(x, None, sv.desc_of(x), r, None, 0, y, None, sv.desc_of(y))
    sv.sv_rope3d_rotate(g, None, sv.desc_of(g), r, None, 1, back, None, sv.desc_of(back))
    torch.cuda.synchronize()
    a, b = float((y.double() * g.double()).sum()), float((x.double() * back.double()).sum())
    size = float((x.abs().double().sum() * g.abs().double().max()) * 4)
    assert abs(a - b) <= size * 4 * E


def test_one_axis_and_capture():
    """Tables of a single axis (the others without pairs, no table given), on another stream and captured: replays follow the buffers."""
    torch = _torch()
    B, H, N, d = 1, 3, 40, 64
    say("rotate one axis, captured")
    q, k = _draw(7, B, H, N, d, "bf16", "bhnd", 2)
    table = wl.rope_tables_3d_factored(N, 1, 1, d)[0]
    full = np.concatenate([table, np.ones((N, d // 2 - table.shape[1], 2), dtype=np.float32)], axis=1)
    cs = torch.from_numpy(np.ascontiguousarray(full)).cuda()
    r = sv.Rope3D(N, 1, 1, d // 2, 0, 0, cs, None, None)
    places = torch.arange(N, dtype=torch.int32, device="cuda")
    positions = torch.stack([places, torch.zeros_like(places), torch.zeros_like(places)], dim=-1).view(B, N, 3).contiguous()
    yq, yk = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.sv_rope3d_rotate(q, k, sv.desc_of(q), r, positions, 0, yq, yk, sv.desc_of(yq), stream=torch.cuda.current_stream())
    for seed in (1, 2, 3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)))
        positions[..., 0] = torch.randperm(N, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        torch.cuda.synchronize()
        want = [torch.empty_like(q) for _ in range(2)]
        other = torch.cuda.Stream()
        sv.sv_rope3d_rotate(q, k, sv.desc_of(q), r, positions, 0, *want, sv.desc_of(q), stream=other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yq, want[0]) and torch.equal(yk, want[1])
        none = np.zeros((1, 0, 2), dtype=np.float32)
        _check(yq, q, (full, none, none), positions.cpu().numpy(), False, "bf16", None, f"q {seed}")


def test_tokens_past_2_gib():
    """Rows 1.3 MiB apart: byte offsets inside a tensor pass 32 bits' sign."""
    torch = _torch()
    N, d, wide = 2100, 64, 655360
    say("rotate rows past 2 GiB")
    big = torch.empty((N, wide), dtype=torch.bfloat16, device="cuda")
    q = big[:, 128:128 + d].unflatten(0, (1, 1, N))
    y = big[:, 1024:1024 + d].unflatten(0, (1, 1, N))
    x, = _draw(9, 1, 1, N, d, "bf16", "bhnd", 1)
    q.copy_(x)
    r = _rope(_tables((21, 10, 10), d))
    sv.sv_rope3d_rotate(q, None, sv.desc_of(q), r, None, 0, y, None, sv.desc_of(y))
    want = torch.empty_like(x)
    sv.sv_rope3d_rotate(x, None, sv.desc_of(x), r, None, 0, want, None, sv.desc_of(want))
    torch.cuda.synchronize()
    assert torch.equal(y, want)
