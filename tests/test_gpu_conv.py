"""The short causal convolution (sv_causal_conv), its token step and its backward pass against 64 bits, within the bounds that
oracle/selective_oracle.py derives."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, ints, like, replayed, same_bits, space, spoil

pytestmark = pytest.mark.gpu

# B, H, N, d, taps, silu, dtype, layout, lengths, cache
CASES = [
    (1, 1, 1, 8, 4, True, "bf16", "bhnd", None, False), (1, 1, 1, 4, 2, False, "f32", "bhnd", None, True),
    (2, 3, 5, 24, 3, True, "bf16", "apart", None, True), (3, 2, 33, 40, 4, False, "bf16", "bnhd", [33, 0, 1], True),
    (4, 5, 21, 112, 4, True, "bf16", "bnhd", [2, 21, 3, 0], False), (4, 5, 21, 112, 3, True, "f32", "apart", [2, 21, 3, 0], True),
    (1, 1, 301, 2240, 4, True, "bf16", "apart", None, True), (2, 1, 67, 264, 2, True, "f32", "bhnd", [67, 66], True),
    (1, 20, 130, 32, 4, True, "bf16", "bhnd", None, True), (7, 8, 150, 128, 3, False, "f32", "bnhd", [150, 0, 1, 75, 149, 96, 128], True),
    (1, 1, 40, 8192, 4, True, "bf16", "bhnd", None, False), (1, 1, 1200, 16, 4, False, "bf16", "bhnd", [1199], True),
    (2, 2, 3000, 64, 4, True, "bf16", "bnhd", [3000, 1601], True),
]


def _id(c):
    return f"{c[0]}x{c[1]}x{c[2]}x{c[3]}-K{c[4]}{'-silu' if c[5] else ''}-{c[6]}-{c[7]}{'-ragged' if c[8] else ''}{'-cache' if c[9] else ''}"


def _inputs(c, seed=1):
    B, H, N, d, K, act, dtype, layout, lengths, cached = c
    x = draw(seed, (B, H, N, d), dtype, layout)
    spoil(x, lengths)
    return x, floats(seed + 1, K, H, d, scale=K ** -0.5), floats(seed + 2, H, d, scale=0.3), draw(seed + 3, (B, H, K - 1, d), dtype) if cached else None


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_forward(c):
    import torch
    B, H, N, d, K, act, dtype, layout, lengths, cached = c
    say(f"conv {_id(c)}")
    x, W, b, cache = _inputs(c)
    want, bound = orc.conv(f64(x), f64(W), f64(b), act, lengths, f64(cache))
    y, out = like(x), torch.full((B, H, K - 1, d), float("nan"), dtype=x.dtype, device="cuda")
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, K, act, ints(lengths), cache, out, y, sv.desc_of(y))
    check("y", y, want["y"], bound["y"], dtype)
    assert np.array_equal(f64(out), want["cache_out"])
    if cached:                                                        # in place, and twice the same bits
        y2 = like(x)
        sv.sv_causal_conv(x, sv.desc_of(x), W, b, K, act, ints(lengths), cache, cache, y2, sv.desc_of(y2))
        same_bits(y, y2)
        same_bits(out, cache)


def test_forward_without_bias_and_cache_out():
    x, W, _, _ = _inputs((2, 2, 19, 48, 4, True, "bf16", "bnhd", None, False))
    want, bound = orc.conv(f64(x), f64(W), None, True)
    y = like(x)
    sv.sv_causal_conv(x, sv.desc_of(x), W, None, 4, 1, None, None, None, y, sv.desc_of(y))
    check("y", y, want["y"], bound["y"], "bf16")


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_backward(c):
    import torch
    B, H, N, d, K, act, dtype, layout, lengths, cached = c
    say(f"conv backward {_id(c)}")
    x, W, b, cache = _inputs(c)
    dy = draw(9, (B, H, N, d), dtype, "bhnd" if layout == "bnhd" else layout)
    spoil(dy, lengths)
    dcache = draw(11, (B, H, K - 1, d), dtype) if cached else None
    # a lane adds up at most 64 tokens, at most 64 lanes' sums are added one after the other, then the workgroups' in sixteen runs
    depth = 64 + 64 + 16 + N * B // 512
    want, bound = orc.conv_backward(f64(x), f64(dy), f64(W), f64(b), act, lengths, f64(cache), f64(dcache), depth)
    ws = space(sv.sv_causal_conv_backward_workspace_bytes(B, H, N, d))
    dx, dc = like(x), torch.full((B, H, K - 1, d), float("nan"), dtype=x.dtype, device="cuda")
    dW, db = torch.full_like(W, float("nan")), torch.full_like(b, float("nan"))
    args = (x, sv.desc_of(x), dy, sv.desc_of(dy), W, b, K, act, ints(lengths), cache, dcache)
    sv.sv_causal_conv_backward(*args, dx, sv.desc_of(dx), dc, dW, db, ws)
    check("dx", dx, want["dx"], bound["dx"], dtype)
    check("dcache_in", dc, want["dcache_in"], bound["dcache_in"], dtype)
    check("dW", dW, want["dW"], bound["dW"], "f32")
    check("db", db, want["db"], bound["db"], "f32")
    dx2, db2 = like(x), torch.full_like(b, float("nan"))              # only some of the gradients
    sv.sv_causal_conv_backward(*args, dx2, sv.desc_of(dx2), None, None, db2, ws)
    same_bits(dx, dx2)
    same_bits(db, db2)
    dx3 = like(x)
    sv.sv_causal_conv_backward(*args, dx3, sv.desc_of(dx3), None, None, None, None)
    same_bits(dx, dx3)


@pytest.mark.parametrize("rows,pool,H,d,K,act,dtype,elsewhere", [
    (1, 1, 1, 8, 4, True, "bf16", False), (5, 9, 3, 40, 2, False, "f32", True), (12, 12, 2, 112, 3, True, "bf16", True), (6, 8, 1, 2240, 4, True, "bf16", False),
    (3, 5, 1, 8192, 4, False, "f32", True)])
def test_token(rows, pool, H, d, K, act, dtype, elsewhere):
    import torch
    say(f"conv token {rows} of {pool} {H}x{d} K{K} {dtype}")
    x = draw(1, (rows, H, 1, d), dtype, "apart")
    W, b = floats(2, K, H, d), floats(3, H, d)
    before = draw(4, (pool, H, K - 1, d), dtype)
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(5))[:rows].tolist()
    if rows > 4:
        order[1], order[2], order[4] = -1, pool, order[0]             # idle, idle, a slot named twice
    cache = before.clone()
    out = torch.full_like(before, float("nan")) if elsewhere else cache
    y = like(x)
    sv.sv_causal_conv_token(x, sv.desc_of(x), W, b, K, act, ints(order), pool, cache, out, y, sv.desc_of(y))
    served, named = f64(y), set()
    expect = np.full((pool, H, K - 1, d), np.nan) if elsewhere else f64(before)
    for r, slot in enumerate(order):
        if not 0 <= slot < pool or slot in named:
            assert np.isnan(served[r]).all()
            continue
        named.add(slot)
        want, bound = orc.conv(f64(x[r:r + 1]), f64(W), f64(b), act, None, f64(before[slot:slot + 1]))
        check("y", y[r:r + 1], want["y"], bound["y"], dtype)
        expect[slot] = want["cache_out"][0]
    assert np.array_equal(f64(out), expect, equal_nan=True)


def test_token_steps_are_a_prompt():
    """Without slots row b works on entry b; nine steps are the prompt's outputs and cache, bit for bit."""
    import torch
    x, W, b, cache = _inputs((3, 2, 9, 64, 4, True, "bf16", "bnhd", None, True))
    y, out = like(x), torch.empty_like(cache)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, 4, 1, None, cache, out, y, sv.desc_of(y))
    steps = like(x)
    for t in range(9):
        sv.sv_causal_conv_token(x[:, :, t:t + 1], sv.desc_of(x[:, :, t:t + 1]), W, b, 4, 1, None, 3, cache, cache, steps[:, :, t:t + 1], sv.desc_of(steps[:, :, t:t + 1]))
    same_bits(y, steps)
    same_bits(out, cache)


def test_a_prompt_in_pieces():
    import torch
    x, W, b, cache = _inputs((2, 1, 50, 72, 4, True, "f32", "bhnd", None, True))
    y, out = like(x), torch.empty_like(cache)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, 4, 1, None, cache, out, y, sv.desc_of(y))
    pieces = like(x)
    for t0, t1 in ((0, 1), (1, 3), (3, 30), (30, 50)):
        part, to = x[:, :, t0:t1], pieces[:, :, t0:t1]
        sv.sv_causal_conv(part, sv.desc_of(part), W, b, 4, 1, None, cache, cache, to, sv.desc_of(to))
    same_bits(y, pieces)
    same_bits(out, cache)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_nonfinite_tokens_stay_where_the_formula_takes_them(value):
    import torch
    c = (1, 1, 60, 64, 4, False, "bf16", "bhnd", None, True)
    x, W, b, cache = _inputs(c)
    y, y2 = like(x), like(x)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, 4, 0, None, cache, None, y, sv.desc_of(y))
    x[0, 0, 30, 5] = value
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, 4, 0, None, cache, None, y2, sv.desc_of(y2))
    differ = (f64(y) != f64(y2))[0, 0]
    assert differ[30:34, 5].all() and differ.sum() == 4 and not np.isfinite(f64(y2)[0, 0, 30:34, 5]).any()
    dy = draw(9, (1, 1, 60, 64), "bf16")
    ws, grads = space(sv.sv_causal_conv_backward_workspace_bytes(1, 1, 60, 64)), []
    x, _, _, _ = _inputs(c)
    for bad in (False, True):
        if bad:
            dy[0, 0, 30, 5] = value
        dx, dW, db = like(x), torch.empty_like(W), torch.empty_like(b)
        sv.sv_causal_conv_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), W, b, 4, 0, None, cache, None, dx, sv.desc_of(dx), None, dW, db, ws)
        grads.append([f64(v) for v in (dx, dW, db)])
    differ = (grads[0][0] != grads[1][0])[0, 0]
    assert differ[27:31, 5].all() and differ.sum() == 4
    assert (grads[0][1] != grads[1][1]).sum() == 4 and (grads[0][2] != grads[1][2]).sum() == 1


def test_a_last_token_that_is_no_number_reaches_its_own_tap_only():
    import torch
    x, W, b, cache = _inputs((2, 1, 70, 16, 4, True, "f32", "bhnd", None, True))
    x[0, 0, 69, 3], x[1, 0, 44, 3] = float("nan"), float("nan")
    dy = draw(9, (2, 1, 70, 16), "f32")
    dx, dW, db = like(x), torch.empty_like(W), torch.empty_like(b)
    ws = space(sv.sv_causal_conv_backward_workspace_bytes(2, 1, 70, 16))
    sv.sv_causal_conv_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), W, b, 4, 0, ints([70, 45]), cache, None, dx, sv.desc_of(dx), None, dW, db, ws)
    assert np.argwhere(np.isnan(f64(dW))).tolist() == [[3, 0, 3]] and not np.isnan(f64(db)).any()
    assert not np.isnan(f64(dx)[0]).any() and not np.isnan(f64(dx)[1, :, :45]).any()


def test_captured_and_replayed():
    import torch
    c = (3, 2, 90, 112, 4, True, "bf16", "bnhd", [90, 17, 0], True)
    x, W, b, cache = _inputs(c)
    dy, dcache, n = draw(9, (3, 2, 90, 112), "bf16", "bnhd"), draw(10, (3, 2, 3, 112), "bf16"), ints([90, 17, 0])
    y, out, dx, dc, dW, db = like(x), torch.empty_like(cache), like(x), torch.empty_like(cache), torch.empty_like(W), torch.empty_like(b)
    ws = space(sv.sv_causal_conv_backward_workspace_bytes(3, 2, 90, 112))
    xd, yd = sv.desc_of(x), sv.desc_of(y)

    def call(stream):
        sv.sv_causal_conv(x, xd, W, b, 4, 1, n, cache, out, y, yd, stream=stream)
        sv.sv_causal_conv_backward(x, xd, dy, sv.desc_of(dy), W, b, 4, 1, n, cache, dcache, dx, sv.desc_of(dx), dc, dW, db, ws, stream=stream)

    def change(i):
        x.copy_(draw(20 + i, (3, 2, 90, 112), "bf16", "bnhd"))
        n.copy_(ints([[90, 17, 0], [3, 90, 44], [1, 2, 90]][i]))
    replayed(call, change, [y, out, dx, dc, dW, db])


def test_rows_of_a_long_tensor_past_32_bits():
    """Tokens 6 MB apart: the last ones lie past 2^31 elements."""
    import torch
    N, stride = 700, 3 << 20
    store = torch.empty(N * stride, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((1, 1, N, 64), (N * stride, N * stride, stride, 1))
    y = store.as_strided((1, 1, N, 64), (N * stride, N * stride, stride, 1), 128)
    x.copy_(draw(1, (1, 1, N, 64), "bf16"))
    W, b = floats(2, 4, 1, 64), floats(3, 1, 64)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, 4, 1, None, None, None, y, sv.desc_of(y))
    want, bound = orc.conv(f64(x), f64(W), f64(b), True)
    check("y", y, want["y"], bound["y"], "bf16")
    ws = space(sv.sv_causal_conv_backward_workspace_bytes(1, 1, N, 64))
    dx, dW, db = like(x.contiguous()), torch.empty_like(W), torch.empty_like(b)
    sv.sv_causal_conv_backward(x, sv.desc_of(x), y, sv.desc_of(y), W, b, 4, 1, None, None, None, dx, sv.desc_of(dx), None, dW, db, ws)
    want, bound = orc.conv_backward(f64(x), f64(y), f64(W), f64(b), True)
    check("dx", dx, want["dx"], bound["dx"], "bf16")
    check("dW", dW, want["dW"], bound["dW"], "f32")
