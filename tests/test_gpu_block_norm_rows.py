"""The gated residual and norms with many rows to a CTA.

A row's results do not depend on its neighbours, so rows of a long call agree
bit for bit with a call on a few of them (which is held to the oracle
elsewhere), wherever the long call's loads of rows ahead wrap around.  Token
sums are compared with float64 on the GPU.  Their bound: float32 sums of at
most 400 terms in sequence (a CTA's rows, then the CTAs' partial sums eight at a
time) lose 400 u = 2.4e-5 of the absolute terms, the terms themselves 1e-5."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# rows and columns: five passes and more to a CTA of 152 SMs' full grid
SHAPES = [(60001, 64), (30011, 120), (20011, 256), (12007, 512), (7001, 520),
          (7001, 1024), (7001, 1536), (4001, 2048), (2003, 4096), (2003, 5120),
          (1009, 8192)]
KINDS = [("layer", "rms", "bf16", "bf16"), ("rms", "layer", "f32", "bf16"),
         ("rms", "rms", "f32", "f32"), ("layer", "none", "bf16", "f32")]
NAMES = ("gate", "scale", "shift", "pre_weight", "post_weight")
A, EPS = 0.75, 1e-5


def _make(rows, dim, kind, seed):
    pre, post, res, blk = kind
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    t = dict(x=(rnd(1, rows, dim) + 1.5).to(DT[res]),
             y=(rnd(1, rows, dim) - 0.5).to(DT[blk]),
             dr=rnd(1, rows, dim).to(DT[res]),
             dh=rnd(1, rows, dim).to(DT[blk]),
             gate=rnd(1, 1, dim), scale=0.4 * rnd(1, 1, dim),
             shift=rnd(1, 1, dim), pre_weight=1 + 0.2 * rnd(dim),
             post_weight=None if post == "none" else 1 + 0.2 * rnd(dim))
    return t


def _parts(rows):
    return [slice(s, s + 37) for s in (0, 41, rows // 2 - 3, rows - 37)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_rows(shape, kind):
    from paper_2609_36757_gb300 import fastvr as FV
    pre, post, res, blk = KINDS[kind]
    t = _make(*shape, KINDS[kind], kind)
    cfg = FV.make_norm_config(pre, post, eps=EPS, residual_scale=A)
    kw = {n: t[n] for n in NAMES}
    r, h = FV.gated_norm(cfg, t["x"], t["y"], **kw)
    for at in _parts(shape[0]):
        few_r, few_h = FV.gated_norm(cfg, t["x"][:, at].contiguous(),
                                     t["y"][:, at].contiguous(), **kw)
        assert torch.equal(few_r, r[:, at]) and torch.equal(few_h, h[:, at])
    # in place
    c = FV._norm_call(cfg, t["x"], (t["y"],), (t["gate"],), ())
    x, h2 = t["x"].clone(), torch.empty_like(h)
    FV.fastvr_gated_norm_fwd(c, x.data_ptr(), t["y"].data_ptr(),
                             *(FV._ptr(kw[n]) for n in NAMES), x.data_ptr(),
                             h2.data_ptr(), FV._stream_of(x))
    assert torch.equal(x, r) and torch.equal(h2, h)


def _unit(v, kind):
    """n(v), rho and the magnitude of n with its cancellation, in float64."""
    mu = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(
        v[..., :1])
    rho = ((v - mu).square().mean(-1, keepdim=True) + EPS).rsqrt()
    return (v - mu) * rho, rho, rho * (v.abs() + mu.abs())


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("shape", SHAPES)
def test_backward_rows(shape, kind):
    from paper_2609_36757_gb300 import fastvr as FV
    pre, post, res, blk = KINDS[kind]
    t = _make(*shape, KINDS[kind], 20 + kind)
    cfg = FV.make_norm_config(pre, post, eps=EPS, residual_scale=A)
    kw = {n: t[n] for n in ("gate", "scale", "pre_weight", "post_weight")}
    got = FV.gated_norm_bwd(cfg, t["dr"], t["dh"], t["x"], t["y"], **kw)
    for at in _parts(shape[0]):
        few = FV.gated_norm_bwd(cfg, *(t[n][:, at].contiguous()
                                       for n in ("dr", "dh", "x", "y")), **kw)
        assert torch.equal(few.dx, got.dx[:, at])
        assert torch.equal(few.dy, got.dy[:, at])
    # the sums over tokens
    f = {n: (None if v is None else v.double()) for n, v in t.items()}
    n, rho, na = _unit(f["x"], pre)
    s1, w = 1 + f["scale"], f["pre_weight"]
    dn = f["dh"] * s1 * w
    avg = lambda v: v.mean(-1, keepdim=True)
    m0 = avg(dn) if pre == "layer" else 0.0
    d = f["dr"] + rho * (dn - m0 - n * avg(dn * n))
    da = f["dr"].abs() + rho * (dn.abs() + avg(dn.abs()) +
                                na * avg(dn.abs() * na))
    u, ua = f["y"], f["y"].abs()
    if post != "none":
        u, _, ua = _unit(f["y"], post)
    pw = 1.0 if f["post_weight"] is None else f["post_weight"]
    ref = dict(dshift=(f["dh"], f["dh"].abs()),
               dscale=(f["dh"] * n * w, f["dh"].abs() * na * w.abs()),
               dpre_weight=(f["dh"] * n * s1, f["dh"].abs() * na * s1.abs()),
               dgate=(d * u * pw, da * ua * (pw if post == "none"
                                             else pw.abs())))
    if post != "none":
        ref["dpost_weight"] = (d * u * f["gate"], da * ua * f["gate"].abs())
    for name, (terms, size) in ref.items():
        want, bound = terms.sum((0, 1)), 4e-5 * size.sum((0, 1)) + 1e-30
        err = (getattr(got, name).double().reshape(-1) - want).abs()
        assert (err <= bound).all(), (name, float((err / bound).max()))
