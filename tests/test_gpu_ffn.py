"""The gated feed-forward on the GPU against the float64 oracle, element by
element.

Bounds, with u = 2^-24 (float32) and r = 2^-8 (bfloat16, half a step):
  g, u_: a float32 sum of D exact products, D u of its absolute terms; saved
      in bfloat16: r of themselves;
  h = act(g) u_: |act'| <= 1.13, so 1.13 |u_| (error of g) + |act| (error of
      u_), 16 u of itself for the activation (exp, erf and tanh to a few u)
      and 16 u |g u_| for it near its zeros, and r of itself;
  dg = dh u_ act'(g): from the saved values, |act''| <= 0.8: 0.8 |dh u_| r |g|
      plus 2 r of itself (u_ saved, dg rounded), 16 u |dh u_|;
  du = dh act(g): 1.13 |dh| r |g| plus r of itself;
  dx, dw: these through their sums, n u of the absolute terms for a float32
      sum of n terms, and r of the result.  Errors of the projections' float32
      sums add to r |g|."""
import numpy as np
import pytest
import torch

from oracle import ffn as OF

pytestmark = pytest.mark.gpu

U, R = 2.0 ** -24, 2.0 ** -8

CASES = [
    # tokens, D, F, activation
    (1, 8, 8, "silu"),
    (1, 1536, 400, "silu"),
    (2, 264, 136, "gelu"),
    (7, 520, 24, "gelu_tanh"),
    (8, 64, 1000, "silu"),
    (16, 1536, 264, "silu"),
    (17, 40, 72, "gelu"),
    (33, 200, 328, "gelu_tanh"),
    (64, 128, 128, "silu"),
    (65, 1000, 120, "gelu"),
    (127, 72, 136, "silu"),
    (128, 64, 256, "gelu_tanh"),
    (129, 320, 128, "silu"),
    (255, 264, 264, "gelu"),
    (257, 8, 640, "silu"),
    (300, 1032, 392, "gelu_tanh"),
    (513, 256, 520, "silu"),
    (1061, 136, 728, "gelu"),
]


def make(case, seed, scale=1.0):
    M, D, F, _ = case
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    bf = lambda t: t.to(torch.bfloat16)
    return (bf(rnd(M, D)), bf(scale * rnd(F, D) * D ** -0.5),
            bf(rnd(F, D) * D ** -0.5), bf(rnd(M, F)))


def n64(t):
    return t.detach().cpu().double().numpy()


def bounds(x, wg, wu, dh, kind):
    x, wg, wu, dh = map(n64, (x, wg, wu, dh))
    M, D = x.shape
    F = wg.shape[0]
    g, u = x @ wg.T, x @ wu.T
    eg = (D + 8) * U * (np.abs(x) @ np.abs(wg).T)
    eu = (D + 8) * U * (np.abs(x) @ np.abs(wu).T)
    a, slope = OF.act(g, kind)
    h = a * u
    b_h = 1.13 * np.abs(u) * eg + np.abs(a) * eu + 16 * U * (
        np.abs(h) + np.abs(g * u)) + R * np.abs(h)
    sg, su = R * np.abs(g) + eg, R * np.abs(u) + eu  # of the saved values
    dg, du = dh * u * slope, dh * a
    edg = 0.8 * np.abs(dh * u) * sg + 1.13 * np.abs(dh) * su + R * np.abs(
        dg) * 1.01 + 16 * U * np.abs(dh * u)
    edu = 1.13 * np.abs(dh) * sg + R * np.abs(du) * 1.01 + 16 * U * np.abs(
        dh * g)
    dx, dwg, dwu = OF.backward(x, wg, wu, dh, kind)
    n = 2 * (F + 8) * U
    b_dx = edg @ np.abs(wg) + edu @ np.abs(wu) + n * (
        np.abs(dg) @ np.abs(wg) + np.abs(du) @ np.abs(wu)) + R * np.abs(dx)
    b_w = []
    for e, t, w in ((edg, dg, dwg), (edu, du, dwu)):
        b_w.append(e.T @ np.abs(x) + (M + 8) * U * (np.abs(t).T @ np.abs(x)) +
                   R * np.abs(w))
    return [(h, b_h), (g, sg), (u, su), (dx, b_dx), (dwg, b_w[0]),
            (dwu, b_w[1])]


def close(got, want, bound, what):
    got = n64(got)
    assert got.shape == want.shape
    err = np.abs(got - want)
    # 1e-38: bfloat16 results below the normal range
    assert (err <= bound * 1.001 + 1e-38).all(), (
        what, float(np.nanmax(err / (bound + 1e-38))))


def check(x, wg, wu, dh, kind, xc=None):
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_ffn_config(kind)
    ref = bounds(x, wg, wu, dh, kind)
    xc = x.cuda() if xc is None else xc
    wg, wu, dh = wg.cuda(), wu.cuda(), dh.cuda()
    h, saved = FV.gated_ffn(cfg, xc, wg, wu, want_saved=True)
    flat = lambda t: t.reshape(-1, t.shape[-1])
    for name, got, r in zip("hgu", (h,) + saved, ref):
        close(flat(got), *r, name)
    # without the projections: the same kernel or another, the same values
    assert torch.equal(h, FV.gated_ffn(cfg, xc, wg, wu))
    g = FV.gated_ffn_bwd(cfg, dh.view(h.shape), xc, wg, wu, saved)
    for name, got, r in zip(g._fields, g, ref[3:]):
        close(flat(got), *r, name)
    frozen = FV.gated_ffn_bwd(cfg, dh.view(h.shape), xc, wg, wu, saved,
                              want_dw=False)
    assert frozen.dw_gate is None and frozen.dw_up is None
    assert torch.equal(frozen.dx, g.dx)
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
    return h, saved, g


@pytest.mark.parametrize("case", CASES, ids=str)
def test_ffn(case):
    check(*make(case, case[0] + case[1]), case[3])


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M", [3, 200])
def test_ffn_saturated_gates(M, kind):
    check(*make((M, 72, 64, kind), 5, 12.0), kind)


@pytest.mark.parametrize("M", [4, 150])
def test_ffn_rows_apart_and_leading_axes(M):
    x, wg, wu, dh = make((2 * M, 64, 136, "silu"), 6)
    wide = torch.full((2 * M, 104), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 16:80] = x.cuda()
    h, _, g = check(x, wg, wu, dh, "silu",
                    wide[:, 16:80].unflatten(0, (2, M)))
    assert h.shape == (2, M, 136) and g.dx.shape == (2, M, 64)
    assert g.dx.is_contiguous()


@pytest.mark.parametrize("M", [2, 260])
def test_ffn_halves_of_a_fused_weight(M):
    x, wg, wu, dh = make((M, 128, 200, "gelu"), 7)
    both = torch.cat([wg, wu]).cuda()
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_ffn_config("gelu")
    assert torch.equal(FV.gated_ffn(cfg, x.cuda(), both[:200], both[200:]),
                       FV.gated_ffn(cfg, x.cuda(), wg.cuda(), wu.cuda()))


@pytest.mark.parametrize("M", [1, 5, 40, 200])
def test_ffn_nan_and_infinity_stay_in_their_rows(M):
    from paper_2609_36757_gb300 import fastvr as FV
    x, wg, wu, _ = make((M, 264, 200, "silu"), 8)
    cfg = FV.make_ffn_config("silu")
    clean = FV.gated_ffn(cfg, x.cuda(), wg.cuda(), wu.cuda())
    for junk in (float("nan"), float("inf")):
        bad = x.clone()
        bad[M // 2, 100] = junk
        h = FV.gated_ffn(cfg, bad.cuda(), wg.cuda(), wu.cuda())
        keep = torch.arange(M) != M // 2
        assert torch.equal(h[keep.cuda()], clean[keep.cuda()])
        assert not bool(torch.isfinite(h[M // 2]).all())


@pytest.mark.parametrize("M", [3, 300])
def test_ffn_repeats_bit_for_bit_and_replays(M):
    from paper_2609_36757_gb300 import fastvr as FV
    x, wg, wu, dh = (t.cuda() for t in make((M, 264, 328, "silu"), 9))
    cfg = FV.make_ffn_config("silu")

    def once():
        h, saved = FV.gated_ffn(cfg, x, wg, wu, want_saved=True)
        return (h,) + tuple(FV.gated_ffn_bwd(cfg, dh, x, wg, wu, saved))

    first = once()
    for a, b in zip(first, once()):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = once()
    x.mul_(0.5)
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


@pytest.mark.parametrize("M", [1, 64, 300])
def test_ffn_writes_nothing_behind_its_outputs(M):
    from paper_2609_36757_gb300 import fastvr as FV
    D, F = 72, 200
    x, wg, wu, dh = (t.cuda() for t in make((M, D, F, "gelu"), 10))
    cfg = FV.make_ffn_config("gelu")
    h, saved = FV.gated_ffn(cfg, x, wg, wu, want_saved=True)
    want = (h,) + saved + tuple(FV.gated_ffn_bwd(cfg, dh, x, wg, wu, saved))
    held = [torch.full((t.numel() + 512,), 7.0, dtype=t.dtype, device="cuda")
            for t in want]
    p = [t.data_ptr() + 512 for t in held]  # 256 elements before and after
    c, row = FV._ffn_call(cfg, x, wg, wu, ())
    n = FV.fastvr_gated_ffn_bwd_scratch_bytes(c)
    scratch = torch.full((n + 512,), 7, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    FV.fastvr_gated_ffn_fwd(c, x.data_ptr(), row, wg.data_ptr(), wu.data_ptr(),
                            *p[:3], stream)
    FV.fastvr_gated_ffn_bwd(c, dh.data_ptr(), x.data_ptr(), row, wg.data_ptr(),
                            wu.data_ptr(), p[1], p[2], *p[3:],
                            scratch.data_ptr() + 256, n, stream)
    for back, t in zip(held, want):
        assert torch.equal(back[256:-256], t.flatten())
        assert bool((back[:256] == 7.0).all() and (back[-256:] == 7.0).all())
    assert bool((scratch[:256] == 7).all() and (scratch[-256:] == 7).all())
