"""Cross attention on the GPU against the float64 oracle, element by element.

Bounds, with u = 2^-24 (float32) and r = 2^-8 (bfloat16, half a step):
  s = scale q.k: products of bfloat16 are exact in float32, a sum of d of them
      is off by at most d u of its absolute terms, the scaling and the exp2
      argument by a few u more: ds = (d + 8) u scale max|q| |k|;
  p:  exp is off by ds plus e = 8e-5, which covers CUDA's exp2 (a few u) and a
      polynomial to 7.5e-5; p enters its products in bfloat16: one r;
  lse: ds, the sum of T terms (T u) and the logarithm (4 u of its magnitude
      and 2^-22);
  out = sum p v / sum p: (r + 2 (ds + e)) sum p |v|, and r of itself;
  D = dout.out takes out as it was rounded: sum |dout| (bound of out);
  dP: d u of its absolute terms;
  dS = p (dP - D), p unrounded here: (r + 2 (ds + e)) of its absolute value
      and p times the errors of dP and D;
  dq, dk, dv: these through their sums, n u of the absolute terms for a
      float32 sum of n terms, and r of the result."""
import numpy as np
import pytest
import torch

from oracle import cross as OC

pytestmark = pytest.mark.gpu

U, R, E = 2.0 ** -24, 2.0 ** -8, 8e-5

CASES = [
    # B, L, T, H, K, d, lens (None: all keys)
    (1, 1, 1, 1, 1, 64, None),
    (1, 1, 77, 12, 12, 128, None),
    (3, 1, 300, 8, 2, 128, [300, 0, 131]),
    (2, 2, 1, 4, 4, 64, [1, 0]),
    (16, 1, 513, 4, 1, 64, list(range(0, 528, 33))),
    (1, 5, 1030, 16, 2, 128, None),
    (2, 4, 129, 6, 3, 64, [128, 129]),
    (1, 2, 1030, 16, 2, 128, None),
    (1, 1, 2000, 2, 1, 64, None),
    (2, 3, 700, 12, 2, 128, [700, 5]),
    (1, 32, 260, 1, 1, 64, None),
    (1, 17, 40, 2, 1, 128, None),
    (2, 127, 128, 3, 3, 128, [1, 128]),
    (1, 128, 129, 2, 2, 64, None),
    (1, 129, 127, 2, 2, 128, None),
    (3, 257, 256, 2, 1, 128, [256, 0, 7]),
    (1, 300, 257, 4, 2, 64, None),
    (2, 385, 512, 2, 2, 128, [385, 512]),
    (5, 130, 333, 4, 1, 64, [-3, 333, 1000, 200, 127]),
    (1, 700, 640, 3, 3, 128, None),
    (2, 1100, 97, 2, 1, 64, [97, 96]),
    # many units to a CTA: one key tile each, and lengths of all kinds
    (3, 1500, 100, 40, 20, 128, None),
    (40, 300, 60, 10, 5, 64, [0, 60, 7, 60] * 10),
    (3, 900, 260, 50, 25, 128, [260, 0, 1]),
    (33, 280, 300, 8, 8, 64, [300, 1, 129] * 11),
    # more entries than lengths are weighed
    (4500, 34, 9, 1, 1, 64, [9, 0, 4] * 1500),
]


def make(case, seed, scale=1.0):
    B, L, T, H, K, d, lens = case
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    q = (scale * rnd(B, L, H, d)).to(torch.bfloat16)
    kv = rnd(B, T, 2 * K, d).to(torch.bfloat16)
    do = rnd(B, L, H, d).to(torch.bfloat16)
    return q, kv[:, :, :K], kv[:, :, K:], do, lens


def n64(t):
    return t.detach().cpu().double().numpy()


def bounds(q, k, v, do, lens, scale):
    """Oracle results and their bounds: (out, lse, dq, dk, dv) pairs."""
    q, k, v, do = map(n64, (q, k, v, do))
    B, L, H, d = q.shape
    T, K = k.shape[1:3]
    G = H // K
    out, lse = OC.forward(q, k, v, lens, scale)
    grads = OC.backward(q, k, v, do, lens, scale)
    b_out, b_lse = np.zeros_like(out), np.zeros_like(lse)
    b_g = [np.zeros_like(t) for t in grads]
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        if n == 0:
            continue
        for h in range(H):
            j = h // G
            kk, vv, qq, g = k[b, :n, j], v[b, :n, j], q[b, :, h], do[b, :, h]
            ds = (d + 8) * U * scale * (np.abs(qq) @ np.abs(kk).T).max(-1)
            ds = ds[:, None]
            p = np.exp(scale * qq @ kk.T - lse[b, h][:, None])
            b_out[b, :, h] = (R + 2 * (ds + E)) * (p @ np.abs(vv)) + \
                R * np.abs(out[b, :, h]) + n * U * (p @ np.abs(vv))
            b_lse[b, h] = ds[:, 0] + n * U + 4 * U * np.abs(lse[b, h]) + \
                2.0 ** -22
            dp = g @ vv.T
            D = (g * out[b, :, h]).sum(-1, keepdims=True)
            s = p * (dp - D)
            es = (R + 2 * (ds + E)) * np.abs(s) + p * (
                (d + 4) * U * (np.abs(g) @ np.abs(vv).T) +
                (np.abs(g) * b_out[b, :, h]).sum(-1, keepdims=True))
            b_g[0][b, :, h] = scale * (es @ np.abs(kk) +
                                       n * U * (np.abs(s) @ np.abs(kk)))
            rows = L * G * U
            b_g[1][b, :n, j] += scale * (es.T @ np.abs(qq) +
                                         rows * (np.abs(s).T @ np.abs(qq)))
            ep = (R + ds + E) * p
            b_g[2][b, :n, j] += ep.T @ np.abs(g) + rows * (p.T @ np.abs(g))
    b_g = [x + R * np.abs(y) for x, y in zip(b_g, grads)]
    return [(out, b_out), (lse, b_lse)] + list(zip(grads, b_g))


def close(got, want, bound, what):
    got = n64(got)
    assert got.shape == want.shape
    same = np.isneginf(got) & np.isneginf(want)
    with np.errstate(invalid="ignore"):
        err = np.where(same, 0.0, np.abs(got - want))
    assert (err <= bound + 1e-30).all(), (
        what, float(np.nanmax(err / (bound + 1e-30))), int((~(err <= bound + 1e-30)).sum()))


def cuda_len(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32,
                                                  device="cuda")


def check(q, k, v, do, lens, scale=0.0, run=None):
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_cross_config(scale)
    ref = bounds(q, k, v, do, lens, scale or q.shape[-1] ** -0.5)
    kv_len = cuda_len(lens)
    qc, kc, vc, gc = (t if t.is_cuda else t.cuda() for t in (q, k, v, do))
    out, lse = FV.cross_attention(cfg, qc, kc, vc, kv_len, want_lse=True)
    close(out, *ref[0], "out")
    close(lse, *ref[1], "lse")
    grads = FV.cross_attention_bwd(cfg, qc, kc, vc, out, gc, lse, kv_len)
    for name, got, r in zip(grads._fields, grads, ref[2:]):
        close(got, *r, name)
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
    return out, lse, grads


@pytest.mark.parametrize("case", CASES, ids=str)
def test_cross(case):
    check(*make(case, 100 + len(str(case))))


@pytest.mark.parametrize("case", [(1, 3, 200, 4, 2, 128, None),
                                  (2, 260, 200, 4, 2, 64, [150, 200])],
                         ids=str)
def test_cross_peaked_and_scaled(case):
    check(*make(case, 7, 3.0), scale=0.4)


@pytest.mark.parametrize("case", [(2, 3, 200, 4, 2, 128, [130, 0]),
                                  (2, 300, 200, 4, 2, 128, [130, 0]),
                                  (2, 300, 300, 2, 2, 64, [256, 129])],
                         ids=str)
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -3e38])
def test_cross_padding_does_not_matter(case, junk):
    q, k, v, do, lens = make(case, 8)
    for b, n in enumerate(lens):
        k[b, n:], v[b, n:] = junk, junk
    clean_k, clean_v = k.clone(), v.clone()
    for b, n in enumerate(lens):
        clean_k[b, n:], clean_v[b, n:] = 0, 0
    from paper_2609_36757_gb300 import fastvr as FV
    cfg, kv_len = FV.make_cross_config(), cuda_len(lens)
    got = []
    for kk, vv in ((k, v), (clean_k, clean_v)):
        t = [x.cuda() for x in (q, kk, vv, do)]
        out, lse = FV.cross_attention(cfg, *t[:3], kv_len, want_lse=True)
        got.append((out, lse) + tuple(FV.cross_attention_bwd(
            cfg, *t[:3], out, t[3], lse, kv_len)))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    check(q, clean_k, clean_v, do, lens)


def strided(t, order):
    """t's values in memory of another order of the first three axes, with gaps
    of junk around every head."""
    shape = [t.shape[i] for i in order] + [t.shape[3] + 8]
    shape[2] += 1
    back = torch.full(shape, float("nan"), dtype=t.dtype, device="cuda")
    view = back[:, :, :t.shape[order[2]], :t.shape[3]]
    inverse = [order.index(i) for i in range(3)] + [3]
    view = view.permute(inverse)
    view.copy_(t)
    return view


@pytest.mark.parametrize("L", [2, 150])
@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (1, 0, 2), (2, 1, 0)])
def test_cross_strides(L, order):
    q, k, v, do, lens = make((2, L, 140, 4, 2, 64, [140, 66]), 9)
    check(*(strided(t, order) for t in (q, k, v, do)), lens)


@pytest.mark.parametrize("L", [1, 200])
def test_cross_outputs_with_strides_leave_the_rest(L):
    from paper_2609_36757_gb300 import fastvr as FV
    q, k, v, do, _ = make((2, L, 140, 4, 2, 64, None), 10)
    q, k, v, do = (t.cuda().contiguous() for t in (q, k, v, do))
    cfg = FV.make_cross_config()
    out, lse = FV.cross_attention(cfg, q, k, v, want_lse=True)
    want = (out,) + tuple(FV.cross_attention_bwd(cfg, q, k, v, out, do, lse))
    c = FV._cross_call(cfg, q, k, v, None)[0]
    # 7.0 around every head of every output
    held, got = [], []
    for t in want:
        back = torch.full(t.shape[:2] + (t.shape[2] + 1, t.shape[3] + 8), 7.0,
                          dtype=t.dtype, device="cuda")
        held.append(back)
        got.append(back[:, :, :t.shape[2], :t.shape[3]])
    s = [FV._head_strides(t, "") for t in got]
    p = [t.data_ptr() for t in got]
    n = FV.fastvr_cross_attn_bwd_scratch_bytes(c)
    scratch = torch.full((n // 4,), float("nan"), device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    FV.fastvr_cross_attn_fwd(c, q.data_ptr(), None, k.data_ptr(), None,
                             v.data_ptr(), None, 0, p[0], s[0], 0, stream)
    FV.fastvr_cross_attn_bwd(c, q.data_ptr(), None, k.data_ptr(), None,
                             v.data_ptr(), None, 0, p[0], s[0], do.data_ptr(),
                             None, lse.data_ptr(), p[1], s[1], p[2], s[2],
                             p[3], s[3], scratch.data_ptr(), n, stream)
    for back, view, t in zip(held, got, want):
        assert torch.equal(view, t)
        view.fill_(7.0)
        assert bool((back == 7.0).all())


@pytest.mark.parametrize("L", [1, 2, 300])
def test_cross_one_prompt_for_the_batch(L):
    q, k, v, do, _ = make((3, L, 190, 4, 2, 128, None), 11)
    k, v = (t[:1].cuda().expand(3, -1, -1, -1) for t in (k, v))
    check(q, k, v, do, [190, 40, 0])


@pytest.mark.parametrize("case", [(2, 1, 700, 8, 2, 128, [700, 300]),
                                  (2, 900, 400, 4, 2, 128, [399, 400])],
                         ids=str)
def test_cross_repeats_bit_for_bit_and_replays(case):
    from paper_2609_36757_gb300 import fastvr as FV
    q, k, v, do, lens = (t.cuda() if torch.is_tensor(t) else t
                         for t in make(case, 12))
    cfg, kv_len = FV.make_cross_config(), cuda_len(lens)

    def once():
        out, lse = FV.cross_attention(cfg, q, k, v, kv_len, want_lse=True)
        return (out, lse) + tuple(
            FV.cross_attention_bwd(cfg, q, k, v, out, do, lse, kv_len))

    first = once()
    for a, b in zip(first, once()):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = once()
    # a replay reads the buffers as they are then, lengths included
    q.mul_(0.5)
    kv_len.copy_(torch.tensor([0, 130], dtype=torch.int32))
    graph.replay()
    want = once()
    for a, b in zip(held, want):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a, b in zip(once(), want):
            assert torch.equal(a, b)
    torch.cuda.synchronize()


def test_cross_rows_are_independent_of_the_path():
    """A call with one query agrees with the same row of a call with many."""
    from paper_2609_36757_gb300 import fastvr as FV
    q, k, v, _, _ = (t.cuda() if torch.is_tensor(t) else t for t in
                     make((1, 400, 500, 8, 2, 128, None), 13))
    cfg = FV.make_cross_config()
    many, lse = FV.cross_attention(cfg, q, k, v, want_lse=True)
    for i in (0, 127, 128, 399):
        one, l1 = FV.cross_attention(cfg, q[:, i:i + 1], k, v, want_lse=True)
        # both within the bound of the formula, so within twice of each other
        torch.testing.assert_close(l1[..., 0], lse[..., i], atol=2e-4, rtol=0)
        torch.testing.assert_close(one[:, 0].float(), many[:, i].float(),
                                   atol=2 * (2 * R + 2 * E) * 4.5, rtol=0)


@pytest.mark.parametrize("case", [(1, 2000, 512, 12, 12, 128, None),
                                  (3, 1100, 130, 16, 4, 64, [130, 64, 2])],
                         ids=str)
def test_cross_bwd_many_times(case):
    """dq's units follow one another without a gap, its warps at their own pace:
    every one of many calls gives the first one's bits and no wait runs out."""
    from paper_2609_36757_gb300 import fastvr as FV
    q, k, v, do, lens = (t.cuda() if torch.is_tensor(t) else t
                         for t in make(case, 14))
    cfg, kv_len = FV.make_cross_config(), cuda_len(lens)
    out, lse = FV.cross_attention(cfg, q, k, v, kv_len, want_lse=True)
    first = FV.cross_attention_bwd(cfg, q, k, v, out, do, lse, kv_len)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(2000):
        got = FV.cross_attention_bwd(cfg, q, k, v, out, do, lse, kv_len)
        for a, b in zip(got, first):
            differ += (a != b).sum()
    assert int(differ) == 0
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK


@pytest.mark.parametrize("at", [0, 4, 8, 12])
@pytest.mark.parametrize("d", [64, 128])
def test_cross_bwd_scratch_on_any_16_bytes(d, at):
    """Split sums in scratch that begins `at` floats past a boundary."""
    from paper_2609_36757_gb300 import fastvr as FV
    q, k, v, do, _ = (t.cuda() if torch.is_tensor(t) else t for t in
                      make((1, 700, 640, 3, 3, d, None), 15))
    k, v = k.contiguous(), v.contiguous()
    cfg = FV.make_cross_config()
    out, lse = FV.cross_attention(cfg, q, k, v, want_lse=True)
    want = FV.cross_attention_bwd(cfg, q, k, v, out, do, lse)
    c = FV._cross_call(cfg, q, k, v, None)[0]
    n = FV.fastvr_cross_attn_bwd_scratch_bytes(c)
    assert n > 2 * 3 * 768 * 4  # there are parts
    back = torch.full((n // 4 + 32,), 7.0, device="cuda")
    scratch = back[at:at + n // 4]
    got = [torch.empty_like(t) for t in want]
    FV.fastvr_cross_attn_bwd(
        c, q.data_ptr(), None, k.data_ptr(), None, v.data_ptr(), None, 0,
        out.data_ptr(), None, do.data_ptr(), None, lse.data_ptr(),
        got[0].data_ptr(), None, got[1].data_ptr(), None, got[2].data_ptr(),
        None, scratch.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    scratch.fill_(7.0)
    assert bool((back == 7.0).all())


@pytest.mark.parametrize("L,d", [(40, 64), (200, 128)])
def test_cross_more_keys_than_are_run_through_at_once(L, d):
    """The forward's loop over key tiles is cut every 1024 tiles; one unit of one
    query tile, one of two, the second batch entry ending at the first cut."""
    T = 1024 * 128 + 130
    check(*make((2, L, T, 1, 1, d, [T, T - 130]), 16))
