"""Gradients of a weight that the gated norm does not use (CPU)."""
import numpy as np

from oracle import block_norm as BN


def test_post_weight_without_a_post_norm():
    """Without a post norm its weight is not used: the forward ignores it and
    its gradient, like that of anything else unused, is zero."""
    g = np.random.default_rng(4)
    B, G, T, D = 2, 3, 2, 16
    L = G * T
    x, y, dr, dh = g.standard_normal((4, B, L, D))
    gate, scale, shift = g.standard_normal((3, B, G, D))
    w = g.standard_normal(D)
    f = lambda w: BN.forward(x, y, gate, scale, shift, None, w, "rms", "none")
    (r, h), (r2, h2) = f(w), f(w + 1.0)
    assert np.array_equal(r, r2) and np.array_equal(h, h2)
    got = BN.backward(dr, dh, r, y, gate, scale, None, w, "rms", "none",
                      groups=G)
    assert got["dpost_weight"].shape == (D,)
    assert (got["dpost_weight"] == 0).all()
    ref = BN.backward(dr, dh, r, y, gate, scale, None, None, "rms", "none",
                      groups=G)
    for name in ("dx", "dy", "dgate", "dscale", "dshift"):
        assert np.array_equal(got[name], ref[name])
