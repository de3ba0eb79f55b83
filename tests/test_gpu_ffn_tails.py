"""The feed-forward's activations far below zero, where they are small: relative
to themselves, not to the gate's value.

Gates and ups are single products of bfloat16 numbers, so exact.  With u = 2^-24
(float32) and r = 2^-8 (bfloat16, half a step), y the activation's argument:
  logistic  1 / (1 + exp(-y)): CUDA gives __expf 2 + 1.173 |y| units of 2u and
      __fdividef two, the sum one more u: (10 + 2.4 |y|) u;
  silu      that with y = g, and u for the product;
  gelu_tanh y = g (c1 + c2 g^2) is off by 4 u of itself, which exp turns into
      4 u |y|: (11 + 6.4 |y|) u;
  gelu      g Phi(g), Phi(-a) = exp(-a^2 / 2) P(t): (4 + 1.2 g^2) u for __expf and
      g^2 / 2 u for its argument, P's fit 10 u, its seven steps 7 u, and t, a
      quotient off by 4 u, as much again, 3 u for products: (28 + 1.7 g^2) u;
and r for the rounded result.  Slopes are sums that may cancel: the same of the
sum's absolute terms, and 4 u where 1 - logistic stands (a difference).  Below
2^-126 float32 holds nothing in full: FLOOR times the other factors."""
import math

import numpy as np
import pytest
import torch

from oracle import ffn as OF

pytestmark = pytest.mark.gpu

U, R, FLOOR = 2.0 ** -24, 2.0 ** -8, 2.0 ** -120
# as far down as the logistic function, or half of erfc, is above 2^-126
LOW = {"silu": -64.0, "gelu": -10.0, "gelu_tanh": -7.875}
F = 264


def n64(t):
    return t.detach().cpu().double().numpy()


def act(g, kind):
    """act(g) and its slope, accurate relative to themselves: (1 + tanh y) / 2 and
    (1 + erf y) / 2 lose that in 64 bits too."""
    if kind == "gelu":
        c = np.vectorize(math.erfc)(-g / math.sqrt(2)) / 2
        return g * c, c + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    y = g if kind == "silu" else 2 * OF._A * (g + OF._B * g ** 3)
    dy = 1.0 if kind == "silu" else 2 * OF._A * (1 + 3 * OF._B * g * g)
    s = 1 / (1 + np.exp(-y))
    return g * s, s + g * dy * s * (1 - s)


def relative(g, kind):
    if kind == "silu":
        return (11 + 2.4 * np.abs(g)) * U
    if kind == "gelu":
        return (28 + 1.7 * g * g) * U
    return (11 + 6.4 * np.abs(2 * OF._A * (g + OF._B * g ** 3))) * U


def gates(kind):
    return torch.linspace(LOW[kind], 6.0, F).to(torch.bfloat16)


def weights(kind):
    wg, wu = (torch.zeros(F, 16, dtype=torch.bfloat16) for _ in range(2))
    wg[:, 0] = gates(kind)
    wu[:, 1] = torch.where(torch.arange(F) % 3 == 0, -1.5, 1.0)
    return wg, wu


@pytest.mark.parametrize("M", [1, 5, 13, 29, 40, 300])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_forward(kind, M):
    from paper_2609_36757_gb300 import fastvr as FV
    wg, wu = weights(kind)
    x = torch.zeros(M, 16, dtype=torch.bfloat16)
    x[:, 0] = 0.75 + 0.5 * (torch.arange(M) % 17) / 16
    x[:, 1] = 1.0
    h = FV.gated_ffn(FV.make_ffn_config(kind), x.cuda(), wg.cuda(), wu.cuda())
    g, u = n64(x) @ n64(wg).T, n64(x) @ n64(wu).T
    a = act(g, kind)[0]
    err = np.abs(n64(h) - a * u)
    bound = (R + relative(g, kind)) * np.abs(a * u) + FLOOR * np.abs(u)
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_slopes(kind):
    """One token with x = 1: dw_gate and dw_up are dg and du themselves."""
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_ffn_config(kind)
    wg, wu = weights(kind)
    x = torch.zeros(1, 16, dtype=torch.bfloat16)
    x[0, :2] = 1.0
    _, saved = FV.gated_ffn(cfg, x.cuda(), wg.cuda(), wu.cuda(),
                            want_saved=True)
    dh = torch.full((1, F), 0.75, dtype=torch.bfloat16)
    got = FV.gated_ffn_bwd(cfg, dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(),
                           saved)
    g, u = n64(wg)[:, 0], n64(wu)[:, 1]
    a, slope = act(g, kind)
    e = relative(g, kind)
    du = 0.75 * a
    err = np.abs(n64(got.dw_up)[:, 0] - du)
    assert (err <= (R + e) * np.abs(du) + FLOOR * (1 + np.abs(g))).all()
    if kind == "gelu":
        rest = np.abs(g) * np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
        terms = np.abs(a / g) + rest
        # exp(-g^2 / 2): 2 + 1.173 g^2 / 2 units of 2 u, 3 u of the argument
        off = (e + (8 + 3 * g * g) * U) * terms
    else:
        s = a / g
        inner = 1.0 if kind == "silu" else 2 * OF._A * (1 + 3 * OF._B * g * g)
        terms = np.abs(s) * (1 + np.abs(g * inner) * (1 - s))
        off = (2 * e + 12 * U) * terms + 4 * U * np.abs(s * g * inner)
    dg = 0.75 * u * slope
    err = np.abs(n64(got.dw_gate)[:, 0] - dg)
    bound = R * np.abs(dg) + 0.75 * np.abs(u) * (
        1.01 * off + FLOOR * (1 + np.abs(g)) ** 3)
    assert (err <= bound).all(), float((err / bound).max())
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
