"""The short causal convolution at the runs of tokens that large calls have, 8 and 16 forwards, 16 to 64 backwards, against 64 bits (tests/test_host_conv_cases.py holds the
library's cuts to the runs named here)."""
import pytest

import paper_2509_24695_amd as sv
from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, ints, like, space, spoil
from tests.test_gpu_conv import _id, _inputs

pytestmark = pytest.mark.gpu

# B, H, N, d, taps, silu, dtype, layout, lengths, cache; tokens of a run
FORWARD = [
    ((2, 1, 2055, 2048, 4, True, "f32", "bhnd", [2055, 1999], True), 8),
    ((3, 1, 2741, 2048, 3, False, "f32", "bnhd", [2741, 17, 2730], True), 16),
    ((2, 9, 5000, 192, 4, True, "bf16", "bnhd", None, False), 8),
]
BACKWARD = [
    ((1500, 1, 600, 16, 4, True, "f32", "bhnd", [600 - b % 601 for b in range(1500)], True), 16),
    ((1100, 1, 1100, 16, 3, True, "bf16", "bhnd", None, False), 32),
    ((2100, 1, 150, 8, 4, False, "bf16", "bnhd", [150 - b % 151 for b in range(2100)], True), 64),
    ((2100, 1, 150, 4, 2, True, "f32", "bhnd", None, True), 64),
]


@pytest.mark.parametrize("c,run", FORWARD, ids=lambda c: _id(c) if isinstance(c, tuple) else f"run{c}")
def test_forward(c, run):
    B, H, N, d, K, act, dtype, layout, lengths, cached = c
    say(f"conv runs {_id(c)}")
    x, W, b, cache = _inputs(c)
    want, bound = orc.conv(f64(x), f64(W), f64(b), act, lengths, f64(cache))
    y = like(x)
    sv.sv_causal_conv(x, sv.desc_of(x), W, b, K, act, ints(lengths), cache, cache, y, sv.desc_of(y))
    check("y", y, want["y"], bound["y"], dtype)
    if cached:
        assert (f64(cache) == want["cache_out"]).all()


@pytest.mark.parametrize("c,run", BACKWARD, ids=lambda c: _id(c) if isinstance(c, tuple) else f"run{c}")
def test_backward(c, run):
    import torch
    B, H, N, d, K, act, dtype, layout, lengths, cached = c
    say(f"conv runs backward {_id(c)}")
    x, W, b, cache = _inputs(c)
    dy = draw(9, (B, H, N, d), dtype, layout)
    spoil(dy, lengths)
    dcache = draw(11, (B, H, K - 1, d), dtype) if cached else None
    # a lane adds up at most 64 tokens, at most 256 lanes' sums are added one after the other, then the workgroups' in sixteen runs
    want, bound = orc.conv_backward(f64(x), f64(dy), f64(W), f64(b), act, lengths, f64(cache), f64(dcache), 64 + 256 + 16 + 4 * B // 16)
    dx, dc = like(x), torch.full((B, H, K - 1, d), float("nan"), dtype=x.dtype, device="cuda")
    dW, db = torch.full_like(W, float("nan")), torch.full_like(b, float("nan"))
    sv.sv_causal_conv_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), W, b, K, act, ints(lengths), cache, dcache, dx, sv.desc_of(dx), dc, dW, db,
                               space(sv.sv_causal_conv_backward_workspace_bytes(B, H, N, d)))
    check("dx", dx, want["dx"], bound["dx"], dtype)
    check("dcache_in", dc, want["dcache_in"], bound["dcache_in"], dtype)
    check("dW", dW, want["dW"], bound["dW"], "f32")
    check("db", db, want["db"], bound["db"], "f32")
