"""Pins of the oracles of rotary positions, gated norms and the 4-bit cache,
and of the library's host-side frequencies (CPU)."""
import math

import numpy as np
import pytest

from oracle import block_norm as BN
from oracle import q4 as Q4
from oracle import rotary as OR


@pytest.fixture(scope="module")
def fv():
    from paper_2609_36757_gb300 import build
    build.build()
    from paper_2609_36757_gb300 import fastvr
    return fastvr


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rotation_keeps_lengths_and_depends_on_relative_positions(layout):
    g = np.random.default_rng(0)
    theta, _ = OR.frequencies([8])
    q, k = g.standard_normal((2, 1, 1, 1, 20))
    at = lambda x, p: OR.rotate(x, [[[p]]], [8], theta, 1.0, layout)
    assert np.isclose(np.linalg.norm(at(q, 7)), np.linalg.norm(q))
    assert np.array_equal(at(q, 7)[..., 16:], q[..., 16:])
    dots = [float((at(q, p + 11) * at(k, p)).sum()) for p in (0, 5, -400)]
    assert np.allclose(dots, dots[0])
    # position 1, first pair: a quarter turn for theta = pi / 2
    one = OR.rotate(np.array([[[[1.0, 0.0]]]]), [[[1]]], [1],
                    np.array([math.pi / 2]), 1.0, layout)
    assert np.allclose(one, [[[[0.0, 1.0]]]])


def test_rotation_transpose_is_the_gradient():
    g = np.random.default_rng(1)
    theta, _ = OR.frequencies([3, 2, 2])
    x, d = g.standard_normal((2, 1, 4, 2, 16))
    pos = g.integers(-50, 50, (1, 4, 3))
    f = lambda x: float((d * OR.rotate(x, pos, [3, 2, 2], theta, 1.3,
                                       "half")).sum())
    grad = OR.rotate(d, pos, [3, 2, 2], theta, 1.3, "half", transpose=True)
    for idx in ((0, 0, 0, 0), (0, 3, 1, 9), (0, 2, 0, 15)):
        e = np.zeros_like(x)
        e[idx] = 0.5
        assert math.isclose(f(x + e) - f(x - e), grad[idx], rel_tol=1e-9)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_library_frequencies_match_the_definition(fv, scaling):
    kw = dict(factors=[4.0, 2.0, 1.0], contexts=[1000, 64, 64])
    theta, mag = OR.frequencies([22, 21, 21], 5000.0, scaling, **kw)
    cfg = fv.make_rotary_config(128, sections=[22, 21, 21], base=5000.0,
                                scaling=scaling, factors=kw["factors"],
                                original_contexts=kw["contexts"])
    got, gmag = fv.fastvr_rotary_frequencies(cfg)
    assert np.allclose(got, theta, rtol=1e-13, atol=0)
    assert math.isclose(gmag, mag, rel_tol=1e-14)


def test_scalings_by_hand(fv):
    plain, _ = OR.frequencies([64])
    ntk, _ = OR.frequencies([64], scaling="ntk", factors=[8.0])
    assert ntk[0] == plain[0] == 1.0
    assert np.isclose(ntk[-1], plain[-1] / 8)   # the slowest: interpolated
    yarn, mag = OR.frequencies([64], scaling="yarn", factors=[8.0],
                               contexts=[4096])
    assert np.isclose(yarn[0], plain[0])        # 652 turns: kept
    assert np.isclose(yarn[-1], plain[-1] / 8)  # 0.07 turns: interpolated
    assert math.isclose(mag, 1 + 0.1 * math.log(8))
    # an explicit magnitude wins
    cfg = fv.make_rotary_config(128, scaling="yarn", factors=[8.0],
                                original_contexts=[4096], magnitude=0.5)
    assert fv.fastvr_rotary_frequencies(cfg)[1] == 0.5


@pytest.mark.parametrize("pre,post", [("rms", "none"), ("layer", "rms"),
                                      ("rms", "layer")])
def test_norm_gradients_match_differences(pre, post):
    g = np.random.default_rng(2)
    B, G, T, D = 2, 3, 2, 16
    L = G * T
    x, y, dr, dh = g.standard_normal((4, B, L, D))
    m = dict(zip(("gate", "scale", "shift"), g.standard_normal((3, B, G, D))))
    w = dict(zip(("pre_weight", "post_weight"), g.standard_normal((2, D))))
    kw = dict(pre=pre, post=post, a=0.8)
    if post == "none":
        w["post_weight"] = None

    def f(x=x, y=y, **over):
        r, h = BN.forward(x, y, **{**m, **w, **over}, **kw)
        return float((dr * r).sum() + (dh * h).sum())

    r, _ = BN.forward(x, y, **m, **w, **kw)
    got = BN.backward(dr, dh, r, y, m["gate"], m["scale"], groups=G, **w, **kw)
    named = dict(dx=("x", x), dy=("y", y), dgate=("gate", m["gate"]),
                 dscale=("scale", m["scale"]), dshift=("shift", m["shift"]),
                 dpre_weight=("pre_weight", w["pre_weight"]),
                 dpost_weight=("post_weight", w["post_weight"]))
    for name, (arg, base) in named.items():
        if base is None:
            continue
        for _ in range(4):
            idx = tuple(g.integers(0, n) for n in base.shape)
            e = np.zeros_like(base)
            e[idx] = 1e-5
            diff = (f(**{arg: base + e}) - f(**{arg: base - e})) / 2e-5
            assert math.isclose(diff, got[name][idx], rel_tol=1e-6,
                                abs_tol=1e-7), name


def test_quantiser_by_hand():
    x = np.zeros(64)
    x[:4] = [7.0, 3.5, -2.5, 0.5]      # s = 1: halves go toward zero
    x[32:36] = [1.0, -1.0, 0.5, 0.07]  # 1/7 = 18.29 / 128: s = 18 / 128
    s = 18 / 128
    want = np.zeros(64)
    want[:4] = [7, 3, -2, 0]
    want[32:36] = [7 * s, -7 * s, 4 * s, 0 * s]  # 0.5 / s = 3.56, 0.07 / s = 0.498
    assert np.array_equal(Q4.values(x), want)
    x[5] = np.inf
    assert np.isnan(Q4.values(x)[:32]).all()
    assert np.array_equal(Q4.values(x)[32:], want[32:])
    assert (Q4.values(np.full(32, 2.0 ** -101)) == 0).all()
    assert np.isnan(Q4.values(np.full(32, 2.0 ** 120))).all()


def _all_bfloat16_pairs():
    """Every (max mantissa, value mantissa, exponent gap) of a group."""
    top, val, gap = np.meshgrid(np.arange(128, 256), np.arange(128, 256),
                                np.arange(0, 6), indexing="ij")
    ok = (gap > 0) | (val <= top)
    return top[ok] / 128.0, val[ok] / 128.0 * 2.0 ** -gap[ok]


def test_quantiser_margins():
    """v / s is an exact half, or at least 2^-14 of itself away from one: a
    reciprocal reduced by 2^-18 therefore gives the definition's rounding in
    float32, and every stored value has 8 significant bits."""
    top, val = _all_bfloat16_pairs()
    s = Q4.scales(top)
    t = val / s
    near = np.abs(t - (np.floor(t) + 0.5))
    assert np.all((near == 0) | (near >= t * 2.0 ** -14))
    r = (np.float32(1 - 2.0 ** -18) / s.astype(np.float32)).astype(np.float32)
    # one fused multiply-add into a float with a unit in the last place of 1
    n32 = np.round(val * r.astype(np.float64))
    assert np.array_equal(np.minimum(n32, 7), np.minimum(np.ceil(t - 0.5), 7))
    assert n32.max() == 7
    for n in range(1, 8):
        m, _ = np.frexp(n * s)
        assert np.all(m * 256 == np.round(m * 256))


def test_attention_oracle_empty_and_shared_heads():
    g = np.random.default_rng(3)
    q = g.standard_normal((2, 4, 8))
    k, v = g.standard_normal((2, 6, 2, 8))
    out, lse, _, _ = Q4.attention(q, k, v, 0.3, np.zeros(6, bool))
    assert (out == 0).all() and (lse == -np.inf).all()
    out, lse, _, _ = Q4.attention(q, k, v, 0.3, np.ones(6, bool))
    s = q[1, 3] @ k[:, 1].T * 0.3
    assert np.isclose(lse[3, 1], np.log(np.exp(s).sum()))
    assert np.allclose(out[1, 3], np.exp(s) @ v[:, 1] / np.exp(s).sum())
