"""CPU oracle for the gated residual and norms -- TEST INFRASTRUCTURE ONLY.

r = a x + gate o post(y),  h = pre(r) o (1 + scale) + shift, in float64, and
the gradients of a scalar sum(dr r) + sum(dh h) written out by the chain rule.
Modulation vectors are [B, G, D]; L / G consecutive tokens share one.

parity pins: tests/test_block_oracle.py -- finite differences of the forward.
"""
import numpy as np


def unit(v, kind, eps):
    """The norm before its weight, and 1 / deviation."""
    if kind == "none":
        return v, np.ones(v.shape[:-1] + (1,))
    if kind == "layer":
        v = v - v.mean(-1, keepdims=True)
    rho = 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    return v * rho, rho


def per_token(m, L, fill):
    if m is None:
        return fill
    return np.repeat(np.asarray(m, np.float64), L // m.shape[1], axis=1)


def forward(x, y, gate=None, scale=None, shift=None, pre_weight=None,
            post_weight=None, pre="rms", post="none", eps=1e-6, a=1.0):
    L = x.shape[1]
    r = a * np.asarray(x, np.float64)
    if y is not None:
        u = unit(np.asarray(y, np.float64), post, eps)[0]
        if post != "none" and post_weight is not None:
            u = u * post_weight
        r = r + per_token(gate, L, 1.0) * u
    h = unit(r, pre, eps)[0]
    if pre_weight is not None:
        h = h * pre_weight
    return r, h * (1 + per_token(scale, L, 0.0)) + per_token(shift, L, 0.0)


def unit_bwd(d, n, rho, kind):
    if kind == "none":
        return d
    g = d - n * (d * n).mean(-1, keepdims=True)
    if kind == "layer":
        g = g - d.mean(-1, keepdims=True)
    return g * rho


def backward(dr, dh, r, y, gate=None, scale=None, pre_weight=None,
             post_weight=None, pre="rms", post="none", eps=1e-6, a=1.0,
             groups=1):
    """dict of dx, dy, dgate, dscale, dshift, dpre_weight, dpost_weight, from
    the stored r; the sums' absolute terms under the same names + "_abs"."""
    r = np.asarray(r, np.float64)
    B, L, D = r.shape
    dr = np.zeros_like(r) if dr is None else np.asarray(dr, np.float64)
    dh = np.zeros_like(r) if dh is None else np.asarray(dh, np.float64)
    w = 1.0 if pre_weight is None else np.asarray(pre_weight, np.float64)
    pw = 1.0 if post_weight is None or post == "none" else np.asarray(
        post_weight, np.float64)
    sc, g = per_token(scale, L, 0.0), per_token(gate, L, 1.0)
    n, rho = unit(r, pre, eps)
    d = dr + unit_bwd(dh * (1 + sc) * w, n, rho, pre)
    out = {"dx": a * d}
    fold = lambda t: t.reshape(B, groups, L // groups, D).sum(2)

    def add(name, terms, how):
        out[name], out[name + "_abs"] = how(terms), how(np.abs(terms))

    everything = lambda t: t.sum((0, 1))
    add("dscale", dh * n * w, fold)
    add("dshift", dh, fold)
    add("dpre_weight", dh * (1 + sc) * n, everything)
    if y is not None:
        yn, ry = unit(np.asarray(y, np.float64), post, eps)
        out["dy"] = unit_bwd(d * g * pw, yn, ry, post)
        add("dgate", d * yn * pw, fold)
        # without a post norm its weight is not used
        add("dpost_weight", d * g * yn if post != "none" else 0.0 * d,
            everything)
    return out
