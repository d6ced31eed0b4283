"""Group norm of more groups than a launch has workgroups of 1 024 threads: each group would fit one, and the call is served all the same."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import selective_oracle as orc
from tests.gpu_util import say
from tests.selective_util import check, draw, f64, floats, like, space

pytestmark = pytest.mark.gpu

H, N, d, G = 131075, 1, 64, 32


def test_forward_and_backward():
    import torch
    say("group norm of 4 194 400 groups")
    x, dy, w, b = draw(1, (1, H, N, d), "bf16"), draw(2, (1, H, N, d), "bf16"), 1 + floats(3, d, scale=0.3), floats(4, d, scale=0.2)
    y, mean, rstd = like(x), torch.full((1, H, G), float("nan"), device="cuda"), torch.full((1, H, G), float("nan"), device="cuda")
    sv.sv_groupnorm(x, sv.desc_of(x), w, b, G, 1e-5, 1, y, sv.desc_of(y), mean, rstd, space(sv.sv_groupnorm_workspace_bytes(1, H, N, d, G)))
    want, bound = orc.group_norm(f64(x), f64(w), f64(b), G, 1e-5, True)
    check("mean", mean, want["mean"], bound["mean"], "f32")
    check("rstd", rstd, want["rstd"], bound["rstd"], "f32")
    check("y", y, want["y"], bound["y"], "bf16")
    stats = [torch.from_numpy(want[k].astype(np.float32)).cuda() for k in ("mean", "rstd")]
    dx, dw, db = like(x), torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    sv.sv_groupnorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, b, G, 1, *stats, dx, sv.desc_of(dx), dw, db, space(sv.sv_groupnorm_backward_workspace_bytes(1, H, N, d, G)))
    # a channel's numbers are added up in sixteen runs
    want, bound = orc.group_norm_backward(f64(x), f64(dy), f64(w), f64(b), G, *map(f64, stats), True, H // 16 + 20)
    check("dx", dx, want["dx"], bound["dx"], "bf16")
    check("dw", dw, want["dw"], bound["dw"], "f32")
    check("db", db, want["db"], bound["db"], "f32")
