"""CPU oracle for cross attention -- TEST INFRASTRUCTURE ONLY.

O = softmax(scale q k^T) v over the first lens[b] keys of batch entry b, in
float64, with query heads sharing key heads in consecutive groups, and the
gradients of sum(dout O) written out by the chain rule.  An entry without keys
gives O = 0, LSE = -inf and no gradients.

parity pins: tests/test_cond_oracle.py -- brute force over scalars, closed
forms, finite differences and planted mistakes.
"""
import numpy as np


def _f(t):
    return np.asarray(t, np.float64)


def forward(q, k, v, lens=None, scale=None):
    """q [B, L, H, d], k and v [B, T, K, d]; (O [B, L, H, d], LSE [B, H, L])."""
    q, k, v = _f(q), _f(k), _f(v)
    B, L, H, d = q.shape
    T, G = k.shape[1], H // k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out, lse = np.zeros_like(q), np.full((B, H, L), -np.inf)
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        if n == 0:
            continue
        for h in range(H):
            s = scale * q[b, :, h] @ k[b, :n, h // G].T
            m = s.max(-1, keepdims=True)
            e = np.exp(s - m)
            z = e.sum(-1, keepdims=True)
            out[b, :, h] = e / z @ v[b, :n, h // G]
            lse[b, h] = (m + np.log(z))[:, 0]
    return out, lse


def backward(q, k, v, dout, lens=None, scale=None):
    """(dq, dk, dv)."""
    q, k, v, dout = _f(q), _f(k), _f(v), _f(dout)
    B, L, H, d = q.shape
    T, G = k.shape[1], H // k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out, lse = forward(q, k, v, lens, scale)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        if n == 0:
            continue
        for h in range(H):
            j = h // G
            p = np.exp(scale * q[b, :, h] @ k[b, :n, j].T - lse[b, h][:, None])
            dp = dout[b, :, h] @ v[b, :n, j].T
            ds = scale * p * (dp - (p * dp).sum(-1, keepdims=True))
            dq[b, :, h] = ds @ k[b, :n, j]
            dk[b, :n, j] += ds.T @ q[b, :, h]
            dv[b, :n, j] += p.T @ dout[b, :, h]
    return dq, dk, dv
