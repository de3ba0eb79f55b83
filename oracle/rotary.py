"""CPU oracle for rotary positions -- TEST INFRASTRUCTURE ONLY.

Plain float64 NumPy from the definition: pair i of an axis with n pairs turns
by p * theta_i, theta_i = base^(-i / n), with the long-context scalings linear
(theta / s), NTK (base * s^(n / (n - 1))) and by-parts (YaRN: pairs that turn
often within the original context keep their frequency, slow ones are divided
by s, a linear ramp between).

parity pins: tests/test_block_oracle.py -- relative positions only, the
transpose is the gradient, hand-evaluated frequencies.
"""
import math

import numpy as np


def frequencies(sections, base=10000.0, scaling="none", factors=None,
                contexts=None, beta_fast=32.0, beta_slow=1.0):
    """theta of every pair, and the default magnitude."""
    theta, biggest = [], 1.0
    for a, n in enumerate(sections):
        s = 1.0 if scaling == "none" else float(factors[a])
        biggest = max(biggest, s)
        for i in range(n):
            b = base
            if scaling == "ntk" and n > 1:
                b = base * s ** (n / (n - 1))
            t = math.exp(-math.log(b) * i / n)
            if scaling == "linear":
                t = t / s
            elif scaling == "yarn":
                turns = contexts[a] * t / (2 * math.pi)
                if turns >= beta_fast:
                    g = 1.0
                elif turns <= beta_slow:
                    g = 0.0
                else:
                    g = (turns - beta_slow) / (beta_fast - beta_slow)
                t = g * t + (1 - g) * t / s
            theta.append(t)
    mag = 0.1 * math.log(biggest) + 1.0 if scaling == "yarn" else 1.0
    return np.array(theta), mag


def rotate(x, positions, sections, theta, magnitude, layout,
           transpose=False):
    """x [B, L, H, d]; positions [B or 1, L, axes] integers."""
    x = np.asarray(x, np.float64)
    axis = np.repeat(np.arange(len(sections)), sections)
    p = np.asarray(positions, np.float64)[..., axis]      # [B, L, pairs]
    # whole turns are dropped in exact integer-friendly arithmetic
    angle = np.remainder(p * theta, 2 * np.pi)[:, :, None, :]
    n = len(theta)
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + n)
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
    if transpose:
        s = -s
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y
