"""The short convolution, the selective scan and the group norm write what they should and nothing else: outputs that are views of larger tensors, workspaces of exactly
the size that is asked for, lengths outside of the rows, calls on two streams at once."""
import pytest

import paper_2509_24695_amd as sv
from tests.gpu_util import say
from tests.selective_util import draw, floats, ints, like, same_bits

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


class _Guarded:
    """Tensors between guards of a byte that nobody writes."""

    def __init__(self):
        self.blocks = []

    def flat(self, nbytes):
        block = _torch().full((nbytes + 8192,), 0xA5, dtype=_torch().uint8, device="cuda")
        self.blocks.append((block, 4096, nbytes))
        return block[4096:4096 + nbytes]

    def dense(self, *shape, dtype=None):
        dtype = dtype or _torch().float32
        n = 1
        for s in shape:
            n *= s
        return self.flat(n * dtype.itemsize).view(dtype).view(shape)

    def rows(self, x):
        """A view [B][H][N][d] of a larger tensor of the guard byte, tokens outside heads, rows apart."""
        B, H, N, d = x.shape
        wide = _torch().full((B * (N + 2) * (H * d + 32) * x.dtype.itemsize,), 0xA5, dtype=_torch().uint8, device="cuda")
        view = wide.view(x.dtype).view(B, N + 2, H * d + 32)[:, 1:N + 1, 16:16 + H * d].unflatten(2, (H, d)).permute(0, 2, 1, 3)
        mask = _torch().ones((B, N + 2, (H * d + 32) * x.dtype.itemsize), dtype=_torch().bool, device="cuda")
        s = x.dtype.itemsize
        self.blocks.append((wide.view(B, N + 2, -1), mask, (N, H * d * s, 16 * s)))
        return view

    def check(self, lengths=None):
        for block, at, size in self.blocks:
            if isinstance(at, int):
                assert (block[:at] == 0xA5).all() and (block[at + size:] == 0xA5).all()
            else:
                N, row, lead = size
                for b in range(block.shape[0]):
                    n = N if lengths is None else max(0, min(N, lengths[b]))
                    inside = at[b].clone()
                    inside[1:1 + n, lead:lead + row] = False
                    assert (block[b][inside] == 0xA5).all()


LENGTHS = [None, [150, -7, 1 << 30]]                                  # values are held to [0, N]
HELD = [150, 0, 150]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", LENGTHS, ids=["whole", "held"])
def test_convolution(dtype, lengths):
    torch = _torch()
    say(f"conv bounds {dtype} {lengths}")
    B, H, N, d, K = 3, 2, 150, 56, 4
    x, dy = draw(1, (B, H, N, d), dtype, "bnhd"), draw(2, (B, H, N, d), dtype, "bnhd")
    W, b, cache = floats(3, K, H, d), floats(4, H, d), draw(5, (B, H, K - 1, d), dtype)
    g = _Guarded()
    y, out = g.rows(x), g.dense(B, H, K - 1, d, dtype=x.dtype)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, K, 1, ints(lengths), cache, out, y, sv.desc_of(y))
    dx, dc, dW, db = g.rows(x), g.dense(B, H, K - 1, d, dtype=x.dtype), g.dense(K, H, d), g.dense(H, d)
    ws = g.flat(sv.sv_causal_conv_backward_workspace_bytes(B, H, N, d))
    sv.sv_causal_conv_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), W, b, K, 1, ints(lengths), cache, cache, dx, sv.desc_of(dx), dc, dW, db, ws)
    torch.cuda.synchronize()
    g.check(lengths)
    held = None if lengths is None else HELD                          # the same as with lengths inside the rows
    y2, out2, dx2, dW2 = like(x), torch.empty_like(cache), like(x), torch.empty_like(W)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, K, 1, ints(held), cache, out2, y2, sv.desc_of(y2))
    sv.sv_causal_conv_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), W, b, K, 1, ints(held), cache, cache, dx2, sv.desc_of(dx2), None, dW2, None, ws)
    same_bits(out, out2)
    same_bits(dW, dW2)
    for i, n in enumerate(held or [N] * B):
        same_bits(y[i, :, :n], y2[i, :, :n])
        same_bits(dx[i, :, :n], dx2[i, :, :n])


@pytest.mark.parametrize("dtype,n", [("bf16", 16), ("f32", 8)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=["whole", "held"])
def test_scan(dtype, n, lengths):
    torch = _torch()
    say(f"scan bounds {dtype} {lengths}")
    B, H, N, d, G = 3, 4, 150, 56, 2
    u, dt, z, dy = (draw(i, (B, H, N, d), dtype, "bnhd") for i in range(4))
    Bm, Cm = draw(5, (B, G, N, n), dtype, "bnhd"), draw(6, (B, G, N, n), dtype, "bnhd")
    A, bias, skip, S, dS = -torch.exp(floats(7, H, d, n)), floats(8, H, d), floats(9, H, d), floats(10, B, H, d, n), floats(11, B, H, d, n)
    g = _Guarded()
    y, s_out = g.rows(u), g.dense(B, H, d, n)
    ws = g.flat(sv.sv_selective_scan_workspace_bytes(B, H, N, d, n))
    ten = (u, dt, sv.desc_of(u), z, sv.desc_of(z), Bm, Cm, sv.desc_of(Bm))
    sv.sv_selective_scan(*ten, A, bias, skip, ints(lengths), S, s_out, y, sv.desc_of(y), ws)
    du, dB = g.rows(u), g.rows(Bm)
    # dU and dDT share u's strides, dB and dC those of Bm: inputs that lie as the guarded outputs do
    wide_u, wide_dt = _Guarded().rows(u).copy_(u), _Guarded().rows(u).copy_(dt)
    wide_B, wide_C, wide_z = _Guarded().rows(Bm).copy_(Bm), _Guarded().rows(Bm).copy_(Cm), _Guarded().rows(u).copy_(z)
    ddt, dz, dC = g.rows(u), g.rows(u), g.rows(Bm)
    grads = [g.dense(B, H, d, n), g.dense(H, d, n), g.dense(H, d), g.dense(H, d)]
    wb = g.flat(sv.sv_selective_scan_backward_workspace_bytes(B, H, N, d, G, n))
    ten = (wide_u, wide_dt, sv.desc_of(wide_u), wide_z, sv.desc_of(wide_z), wide_B, wide_C, sv.desc_of(wide_B))
    sv.sv_selective_scan_backward(*ten, dy, sv.desc_of(dy), A, bias, skip, ints(lengths), S, dS, du, ddt, dz, dB, dC, *grads, wb)
    torch.cuda.synchronize()
    g.check(lengths)
    if lengths is not None:
        y2, s2, dA2 = like(u), torch.empty_like(S), torch.empty_like(A)
        sv.sv_selective_scan(u, dt, sv.desc_of(u), z, sv.desc_of(z), Bm, Cm, sv.desc_of(Bm), A, bias, skip, ints(HELD), S, s2, y2, sv.desc_of(y2), ws)
        sv.sv_selective_scan_backward(*ten, dy, sv.desc_of(dy), A, bias, skip, ints(HELD), S, dS, du, ddt, dz, dB, dC, None, dA2, None, None, wb)
        same_bits(s_out, s2)
        same_bits(grads[1], dA2)
        for i, m in enumerate(HELD):
            same_bits(y[i, :, :m], y2[i, :, :m])


@pytest.mark.parametrize("B,H,N,d,G", [(2, 3, 150, 48, 6), (1, 2, 2500, 296, 4), (1, 2, 2500, 320, 32), (1, 2, 7000, 24, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_group_norm(dtype, B, H, N, d, G):
    torch = _torch()
    say(f"group norm bounds {dtype} {B}x{H}x{N}x{d}-{G}")
    x, dy, w, b = draw(1, (B, H, N, d), dtype, "bnhd"), draw(2, (B, H, N, d), dtype, "bnhd"), floats(3, d), floats(4, d)
    g = _Guarded()
    y, mean, rstd = g.rows(x), g.dense(B, H, G), g.dense(B, H, G)
    ws = g.flat(sv.sv_groupnorm_workspace_bytes(B, H, N, d, G))
    sv.sv_groupnorm(x, sv.desc_of(x), w, b, G, 1e-5, 1, y, sv.desc_of(y), mean, rstd, ws)
    dx, dw, db = g.rows(x), g.dense(d), g.dense(d)
    wb = g.flat(sv.sv_groupnorm_backward_workspace_bytes(B, H, N, d, G))
    sv.sv_groupnorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, b, G, 1, mean, rstd, dx, sv.desc_of(dx), dw, db, wb)
    torch.cuda.synchronize()
    g.check()


def test_calls_on_two_streams():
    """Two scans and two group norms at once, a workspace each, give what they give alone."""
    torch = _torch()
    say("two streams")
    B, H, N, d, n = 2, 1, 900, 640, 16
    sets = []
    for k in range(2):
        u, dt, z, dy = (draw(10 * k + i, (B, H, N, d), "bf16") for i in range(4))
        Bm, Cm = draw(10 * k + 5, (B, 1, N, n), "bf16"), draw(10 * k + 6, (B, 1, N, n), "bf16")
        A, S = -torch.exp(floats(10 * k + 7, H, d, n)), floats(10 * k + 8, B, H, d, n)
        space = lambda nbytes: torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        ws, wg = space(sv.sv_selective_scan_workspace_bytes(B, H, N, d, n)), space(sv.sv_groupnorm_workspace_bytes(B, H, N, d, 8))
        wb = space(sv.sv_selective_scan_backward_workspace_bytes(B, H, N, d, 1, n))

        def run(stream, u=u, dt=dt, z=z, dy=dy, Bm=Bm, Cm=Cm, A=A, S=S, ws=ws, wg=wg, wb=wb):
            y, s, x, du, ddt, dz, dB, dC, dA = (torch.empty_like(v) for v in (u, S, u, u, u, u, Bm, Cm, A))
            D, C = sv.desc_of(u), sv.desc_of(Bm)
            sv.sv_groupnorm(u, D, None, None, 8, 1e-5, 1, x, D, None, None, wg, stream=stream)
            sv.sv_selective_scan(x, dt, D, z, D, Bm, Cm, C, A, None, None, None, S, s, y, D, ws, stream=stream)
            sv.sv_selective_scan_backward(x, dt, D, z, D, Bm, Cm, C, dy, D, A, None, None, None, S, None, du, ddt, dz, dB, dC, None, dA, None, None, wb, stream=stream)
            return y, s, du, ddt, dz, dB, dC, dA
        sets.append(run)
    torch.cuda.synchronize()
    alone = [run(None) for run in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    both = []
    for run, stream in zip(sets, streams):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            both.append(run(stream))
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for x, y in zip(a, b):
            same_bits(x, y)
