"""The chunk by chunk form of the decayed attention's oracle gives what its token by token form gives, results and magnitudes."""
import numpy as np
import pytest

from oracle import decay_oracle as orc


@pytest.mark.parametrize("N,chunk,lengths,state", [(1, 8, None, True), (37, 8, None, False), (64, 16, [64, 0, 1], True), (50, 64, [17, 50, 33], True)])
def test_chunks_are_tokens(N, chunk, lengths, state):
    rng = np.random.default_rng(5)
    B, H, d = 3, 4, 6
    q, k, v, do = rng.standard_normal((4, B, H, N, d))
    s_in, ds_out = rng.standard_normal((2, B, H, d, d)) if state else (None, None)
    g = np.array([0.0, -0.01, -1.3, 0.02])
    n = np.full(B, N) if lengths is None else np.asarray(lengths)
    for x in (q, k, v, do):
        for b in range(B):
            x[b, :, n[b]:] = 0.0
    rows = np.broadcast_to((np.arange(N)[None, :] < n[:, None])[:, None, :, None], q.shape)
    for one, other in ((orc.forward(q, k, v, g, 0.7, s_in, lengths), orc.forward_in_chunks(q, k, v, g, 0.7, s_in, lengths, chunk)),
                       (orc.backward(q, k, v, do, g, 0.7, s_in, ds_out, lengths), orc.backward_in_chunks(q, k, v, do, g, 0.7, s_in, ds_out, lengths, chunk))):
        for a, b in zip(one, other):
            for name in a:
                x = np.where(rows, a[name], 0.0) if a[name].shape == q.shape else a[name]
                assert np.allclose(x, b[name], rtol=1e-12, atol=1e-12), name
