"""Single tokens of more rows than a workgroup has lanes: a slot that an early row has named is found however far behind the other is."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from tests.gpu_util import say, to_host
from tests.test_gpu_decay import E, U, _decays, _draw, _host, _ints, _like, _states, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,dtype,H", [(32, "bf16", 1), (64, "f32", 2), (112, "bf16", 1), (128, "f32", 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_slots_named_twice_far_apart(d, dtype, H, in_place):
    """Bound: two roundings per element of the state, d + 2 of the output's sum, and the output's own."""
    torch = _torch()
    rows, pool = 901, 950
    say(f"decay rows d={d} {dtype} in_place={in_place}")
    q, k, v = _draw(161, rows, H, 1, d, dtype, "packed", 3)
    g, scale = _decays(H), 0.3
    S = _states(22, pool, H, d, d)
    slots = np.random.default_rng(4).permutation(pool)[:rows]
    for late, early in ((300, 0), (555, 299), (899, 255), (900, 256), (900, 898), (700, 0)):
        slots[late] = slots[early]
    slots[[5, 600]] = [pool, -7]
    first = {}
    for r, s in enumerate(slots):
        first.setdefault(int(s), r)
    serves = np.array([first[int(s)] == r and 0 <= s < pool for r, s in enumerate(slots)])
    s_in = S.clone()
    s_out = s_in if in_place else torch.full_like(S, 7.0)
    o = _like(q, 7.0)
    sv.sv_decay_linattn_token(q, k, v, sv.desc_of(q), g, _ints(slots.tolist()), pool, scale, s_in, s_out, o, sv.desc_of(o))
    torch.cuda.synchronize()
    at = slots[serves]
    before, got_s, got_o = _host(S), _host(s_out), _host(o)[:, :, 0]
    qh, kh, vh = (_host(x)[serves, :, 0] for x in (q, k, v))
    kv, l = kh[..., :, None] * vh[..., None, :], np.exp(_host(g))[None, :, None, None]
    want, size = l * before[at] + kv, l * np.abs(before[at]) + np.abs(kv)
    assert (np.abs(got_s[at] - want) <= 4 * E * size).all()
    out, mag = scale * (qh[..., None] * want).sum(2), scale * (np.abs(qh)[..., None] * size).sum(2)
    assert (np.abs(got_o[serves] - out) <= (U if dtype == "bf16" else E) * np.abs(out) + (d + 8) * E * mag).all()
    assert (got_o[~serves] == 7.0).all() and (~serves).sum() == 7
    others = np.setdiff1d(np.arange(pool), at)
    assert np.array_equal(got_s[others], before[others] if in_place else np.full_like(before[others], 7.0))
    assert to_host(s_in).shape == (pool, H, d, d) and (in_place or torch.equal(s_in, S))
