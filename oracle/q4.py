"""CPU oracle for the 4-bit KV cache -- TEST INFRASTRUCTURE ONLY.

From the definition, in exact rational arithmetic on the bfloat16 inputs'
float64 values: a group of 32 consecutive values has s = max |v| / 7 rounded to
5 significant bits (ties to even) and stands for n s, n the whole number
nearest to v / s with ties toward zero, |n| <= 7.  Groups below 2^-100 are
zeros; groups with a NaN, an infinity or a magnitude of 2^120 or more are NaN.
"""
import numpy as np

from . import attention as OA


def scales(top):
    """Scales of groups with max |v| = top (float64, finite, >= 2^-100)."""
    m, e = np.frexp(top)              # top = m 2^e, m in [1/2, 1)
    m = (m * 256).astype(np.int64)    # 8 significant bits: whole numbers
    assert np.all(m / 256.0 * np.exp2(e) == top)
    # top / 7 = (m / 7) 2^(e - 8); five bits of m / 7 = 18.3 .. 36.4: below 32
    # its whole part has 5 bits, from 32 on 6, of which the last is dropped
    def nearest_even(num, den):
        q, r = num // den, num % den
        up = (2 * r > den) | ((2 * r == den) & (q % 2 == 1))
        return q + up
    small = m < 224                   # m / 7 < 32
    q = np.where(small, nearest_even(m, 7), 2 * nearest_even(m, 14))
    return q * np.exp2(e - 8.0)


def values(x):
    """The values that the cache holds for x [..., d] (bfloat16 values)."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    with np.errstate(invalid="ignore"):
        top = np.abs(g).max(-1)
        bad = ~(top < 2.0 ** 120)
        zero = top < 2.0 ** -100
    s = scales(np.where(bad | zero, 1.0, top))[..., None]
    t = np.abs(np.where((bad | zero)[..., None], 0.0, g)) / s
    # halves are exact in float64: v has 8 bits and s 5
    n = np.minimum(np.ceil(t - 0.5), 7)
    out = np.sign(np.where(np.isnan(g), 0, g)) * n * s
    out = np.where(zero[..., None], 0.0, out)
    out = np.where(bad[..., None], np.nan, out)
    return out.reshape(x.shape)


def attention(q, k, v, scale, visible):
    """q [n, H, d], k and v [T, Hkv, d] (cache values), visible [T] bool.
    Returns out [n, H, d], lse [H, n], sum p |v| [n, H, d] and max |score|
    [H, n]."""
    n, H, d = q.shape
    G = H // k.shape[1]
    out, mass = np.zeros((n, H, d)), np.zeros((n, H, d))
    lse, top = np.full((H, n), -np.inf), np.zeros((H, n))
    if not visible.any():
        return out, lse, mass, top
    for h in range(H):
        kk, vv = k[visible, h // G], v[visible, h // G]
        s = (q[:, h] @ kk.T) * scale
        m = s.max(-1, keepdims=True)
        p = np.exp(s - m)
        z = p.sum(-1, keepdims=True)
        out[:, h] = p @ vv / z
        mass[:, h] = p @ np.abs(vv) / z
        lse[h] = (m + np.log(z))[:, 0]
        top[h] = np.abs(s).max(-1)
    return out, lse, mass, top


def visible_tokens(chunks, last_frames, N, k, W, first_chunk=None):
    """Chunk index of every token that chunk chunks - 1 can see, oldest
    first, and whether it is visible to an entry that joined at
    first_chunk."""
    c = chunks - 1
    idx = []
    for cc in OA.visible_chunks(c, W):
        idx += [cc] * ((last_frames if cc == c else k) * N)
    idx = np.array(idx)
    return idx, (np.ones(len(idx), bool) if first_chunk is None
                 else idx >= first_chunk)
