"""Pins of the oracles for cross attention and the gated feed-forward (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import cross as OC
from oracle import ffn as OF


def _draw(seed, B=2, L=3, T=4, H=4, K=2, d=5):
    r = np.random.default_rng(seed)
    return (r.standard_normal((B, L, H, d)), r.standard_normal((B, T, K, d)),
            r.standard_normal((B, T, K, d)), r.standard_normal((B, L, H, d)))


def test_cross_brute_force():
    q, k, v, _ = _draw(0)
    lens = [3, 4]
    out, lse = OC.forward(q, k, v, lens, 0.7)
    for b in range(2):
        for i in range(3):
            for h in range(4):
                s = [0.7 * sum(float(q[b, i, h, x]) * float(k[b, t, h // 2, x])
                               for x in range(5)) for t in range(lens[b])]
                z = math.fsum(map(math.exp, s))
                assert abs(lse[b, h, i] - math.log(z)) < 1e-12
                for x in range(5):
                    o = math.fsum(math.exp(s[t]) * v[b, t, h // 2, x]
                                  for t in range(lens[b])) / z
                    assert abs(out[b, i, h, x] - o) < 1e-12


def test_cross_closed_forms():
    q, k, v, g = _draw(1)
    out, lse = OC.forward(0 * q, k, v, [2, 0])
    np.testing.assert_allclose(out[0, 1, 3], v[0, :2, 1].mean(0))
    np.testing.assert_allclose(lse[0], math.log(2))
    assert (out[1] == 0).all() and np.isneginf(lse[1]).all()
    grads = OC.backward(q, k, v, g, [1, 0])
    assert all((t[1] == 0).all() for t in grads)
    # one key: the output is its value, whatever the query
    assert np.abs(grads[0]).max() < 1e-15 and np.abs(grads[1]).max() < 1e-15
    np.testing.assert_allclose(grads[2][0, 0, 0], g[0, :, :2].sum((0, 1)))
    # padding, and lengths past both ends
    bad_k, bad_v = k.copy(), v.copy()
    bad_k[0, 3:], bad_v[0, 3:] = np.nan, np.inf
    for x, y in zip(OC.forward(q, k, v, [3, 9]),
                    OC.forward(q, bad_k, bad_v, [3, 4])):
        np.testing.assert_array_equal(x, y)
    assert (OC.forward(q, k, v, [-2, 4])[0][0] == 0).all()


def _difference(f, x, i, eps=1e-5):
    up, down = x.copy(), x.copy()
    up.flat[i] += eps
    down.flat[i] -= eps
    return (f(up) - f(down)) / (2 * eps)


def test_cross_gradients_are_differences():
    q, k, v, g = _draw(2)
    lens = [4, 2]
    got = OC.backward(q, k, v, g, lens, 0.6)
    at = [q, k, v]
    for n in range(3):
        f = lambda x: (OC.forward(*(at[:n] + [x] + at[n + 1:]), lens,
                                  0.6)[0] * g).sum()
        for i in range(0, at[n].size, 7):
            assert abs(got[n].flat[i] - _difference(f, at[n], i)) < 1e-7


def test_cross_planted_mistakes_differ():
    q, k, v, g = _draw(3)
    out, _ = OC.forward(q, k, v, [3, 4])
    dq, dk, dv = OC.backward(q, k, v, g, [3, 4])
    far = lambda a, b: np.abs(a - b).max() > 1e-2
    assert far(out, OC.forward(q, k, v, [4, 4])[0])      # padding seen
    assert far(out, OC.forward(q, k, v, [3, 4], 1.0)[0])  # scale dropped
    assert far(out, OC.forward(q, v, k, [3, 4])[0])       # k and v exchanged
    # key heads by turns instead of in groups
    assert far(out, OC.forward(q[:, :, [0, 2, 1, 3]], k, v, [3, 4])[0][
        :, :, [0, 2, 1, 3]])
    # heads of a group not summed
    half = OC.backward(q[:, :, ::2], k, v, g[:, :, ::2], [3, 4])
    assert far(dk, half[1]) and far(dv, half[2])


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_ffn_against_torch_and_differences(kind):
    r = np.random.default_rng(4)
    x, wg, wu = (r.standard_normal(s) for s in ((3, 6), (5, 6), (5, 6)))
    dh = r.standard_normal((3, 5))
    f = torch.nn.functional
    act = {"silu": f.silu, "gelu": f.gelu,
           "gelu_tanh": lambda t: f.gelu(t, approximate="tanh")}[kind]
    t = [torch.tensor(a) for a in (x, wg, wu)]
    ref = act(t[0] @ t[1].T) * (t[0] @ t[2].T)
    np.testing.assert_allclose(OF.forward(x, wg, wu, kind), ref.numpy(),
                               rtol=1e-12, atol=1e-14)
    got, at = OF.backward(x, wg, wu, dh, kind), [x, wg, wu]
    for n in range(3):
        loss = lambda y: (OF.forward(*(at[:n] + [y] + at[n + 1:]), kind) *
                          dh).sum()
        for i in range(at[n].size):
            assert abs(got[n].flat[i] - _difference(loss, at[n], i)) < 1e-6


def test_ffn_closed_forms_and_planted_mistakes():
    a, slope = OF.act(np.array([0.0, 40.0, -40.0]), "silu")
    np.testing.assert_allclose(a, [0, 40, 0], atol=1e-15)
    np.testing.assert_allclose(slope, [0.5, 1, 0], atol=1e-15)
    for kind in ("gelu", "gelu_tanh"):
        a, slope = OF.act(np.array([0.0, 9.0, -9.0]), kind)
        np.testing.assert_allclose(a, [0, 9, 0], atol=1e-14)
        np.testing.assert_allclose(slope, [0.5, 1, 0], atol=1e-13)
    r = np.random.default_rng(5)
    x, wg, wu = (r.standard_normal(s) for s in ((3, 6), (5, 6), (5, 6)))
    h = OF.forward(x, wg, wu, "silu")
    far = lambda b: np.abs(h - b).max() > 1e-2
    assert far(OF.forward(x, wu, wg, "silu")) and far(
        OF.forward(x, wg, wu, "gelu")) and far((x @ wg.T) * (x @ wu.T))
    dh = r.standard_normal((3, 5))
    dx, dwg, dwu = OF.backward(x, wg, wu, dh, "silu")
    assert np.abs(dwg - dwu).max() > 1e-2
