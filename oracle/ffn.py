"""CPU oracle for the gated feed-forward -- TEST INFRASTRUCTURE ONLY.

h = act(x Wg^T) o (x Wu^T) in float64 and the gradients of sum(dh h) written
out by the chain rule.

parity pins: tests/test_cond_oracle.py -- closed forms, torch's activations,
finite differences and planted mistakes.
"""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])
_A, _B = math.sqrt(2 / math.pi), 0.044715


def act(g, kind):
    """act(g) and act'(g)."""
    g = np.asarray(g, np.float64)
    if kind == "silu":
        s = 1 / (1 + np.exp(-g))
        return g * s, s + g * s * (1 - s)
    if kind == "gelu":
        c = (1 + _erf(g / math.sqrt(2))) / 2
        return g * c, c + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    t = np.tanh(_A * (g + _B * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g / 2 * (1 - t * t) * _A * (
        1 + 3 * _B * g * g)


def forward(x, wg, wu, kind):
    x, wg, wu = (np.asarray(t, np.float64) for t in (x, wg, wu))
    return act(x @ wg.T, kind)[0] * (x @ wu.T)


def backward(x, wg, wu, dh, kind):
    """(dx, dwg, dwu)."""
    x, wg, wu, dh = (np.asarray(t, np.float64) for t in (x, wg, wu, dh))
    g, u = x @ wg.T, x @ wu.T
    a, slope = act(g, kind)
    dg, du = dh * u * slope, dh * a
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x
