"""Layer norm's gradients with infinities in them: each reaches the sums that it is a term of, once, and as the formulas have it."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from oracle import layer_oracle as orc
from tests.gpu_util import say, to_host
from tests.test_gpu_norm import _like, _params, _rows, _space, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,dtype", [(32, "f32"), (64, "bf16"), (320, "bf16"), (512, "f32"), (1504, "bf16")])
@pytest.mark.parametrize("in_place", [False, True])
def test_an_infinite_gradient_of_the_last_row(d, dtype, in_place):
    """Rows that do not fill a workgroup.  An infinity in the last row's gradient makes that row's dx NaN or infinite, and its feature of dw and db an
    infinity of its own sign; nothing else."""
    torch = _torch()
    B, H, N = 1, 1, 5
    say(f"norm nonfinite d={d} {dtype} in_place={in_place}")
    x, dy = _rows(1, B, H, N, d, dtype, "bhnd", 0.3), _rows(3, B, H, N, d, dtype, "bhnd", 0.1)
    w, _ = _params(2, 1, d)
    _, mean, rstd = orc.norm(to_host(x), None, None, 1e-5)
    dy[0, 0, -1, 3] = float("inf")
    mean, rstd = (torch.from_numpy(t.astype(np.float32)).cuda() for t in (mean, rstd))
    xh = float(x[0, 0, -1, 3]) - float(mean[0, 0, -1])
    dx, dw, db = dy if in_place else _like(x, 7.0), torch.full((1, d), 7.0, device="cuda"), torch.full((1, d), 7.0, device="cuda")
    sv.sv_layernorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, 1, mean, rstd, dx, sv.desc_of(dx), dw, db, _space(B, H, N, d))
    torch.cuda.synchronize()
    dw, db, dx = to_host(dw)[0], to_host(db)[0], to_host(dx)
    assert dw[3] == np.copysign(np.inf, xh) and db[3] == np.inf
    assert np.isfinite(np.delete(dw, 3)).all() and np.isfinite(np.delete(db, 3)).all()
    assert np.isfinite(dx[0, 0, :-1]).all() and not np.isfinite(dx[0, 0, -1]).any()


@pytest.mark.parametrize("d,dtype", [(32, "f32"), (64, "bf16"), (1504, "bf16")])
def test_an_infinite_weight_in_place(d, dtype):
    """dX over dY with an infinite weight: every dx is NaN or infinite, dw and db are sums of finite numbers."""
    torch = _torch()
    B, H, N = 2, 3, 7
    say(f"norm infinite weight d={d} {dtype}")
    x, dy = _rows(1, B, H, N, d, dtype, "bhnd", 0.3), _rows(3, B, H, N, d, dtype, "bhnd", 0.1)
    w = torch.ones((1, d), device="cuda")
    w[0, 1] = float("inf")
    _, mean, rstd = orc.norm(to_host(x), None, None, 1e-5)
    ref, mag = orc.norm_backward(to_host(x), to_host(dy), None, mean, rstd, False)
    mean, rstd = (torch.from_numpy(t.astype(np.float32)).cuda() for t in (mean, rstd))
    dw, db = torch.full((1, d), 7.0, device="cuda"), torch.full((1, d), 7.0, device="cuda")
    sv.sv_layernorm_backward(x, sv.desc_of(x), dy, sv.desc_of(dy), w, 1, mean, rstd, dy, sv.desc_of(dy), dw, db, _space(B, H, N, d))
    torch.cuda.synchronize()
    bound = 2.0 ** -24 * (B * H * N / 32 + 80)
    assert (np.abs(to_host(dw) - ref["dw"]) <= bound * mag["dw"]).all() and (np.abs(to_host(db) - ref["db"]) <= bound * mag["db"]).all()
