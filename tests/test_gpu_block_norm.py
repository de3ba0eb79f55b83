"""The gated residual and norms on the GPU against the float64 oracle.

Bounds, with u = 2^-24: a sum over D <= 8192 terms in registers, shuffles and
at most 32 partials adds less than 60 u of its absolute terms, the square root
and products a few more; centring x loses u of |x| + |mean|.  So each float32
result is within 1e-5 of its absolute terms (about 170 u); a bfloat16 result
adds 2^-8 of itself.  Token sums run over at most 400 tokens in sequence:
400 u = 2.4e-5, and their terms' own 1e-5."""
import numpy as np
import pytest
import torch

from oracle import block_norm as BN

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CASES = [
    # B, G, tokens of a group, D, pre, post, residual, block
    (1, 1, 1, 8, "rms", "none", "bf16", "bf16"),
    (1, 1, 1, 1536, "layer", "rms", "bf16", "bf16"),
    (2, 3, 5, 264, "layer", "layer", "f32", "bf16"),
    (1, 2, 301, 64, "rms", "rms", "f32", "f32"),
    (3, 1, 129, 520, "layer", "none", "bf16", "f32"),
    (1, 700, 1, 128, "rms", "layer", "bf16", "bf16"),  # a vector per token
    (2, 2, 33, 1032, "rms", "rms", "bf16", "bf16"),
    (1, 3, 40, 2048, "layer", "rms", "f32", "bf16"),
    (1, 2, 9, 4096, "rms", "layer", "bf16", "bf16"),
    (1, 1, 7, 4104, "layer", "rms", "f32", "f32"),
    (2, 1, 3, 8192, "layer", "layer", "bf16", "f32"),
]


def _make(case, seed):
    B, G, T, D, pre, post, res, blk = case
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    L = G * T
    big = torch.where(torch.rand(D, generator=g) < 0.05, 12.0, 1.0)
    t = dict(x=(rnd(B, L, D) * big + 2.0).to(DT[res]),
             y=(rnd(B, L, D) - 0.5).to(DT[blk]), gate=rnd(B, G, D),
             scale=0.4 * rnd(B, G, D), shift=rnd(B, G, D),
             pre_weight=1 + 0.2 * rnd(D), post_weight=1 + 0.2 * rnd(D),
             dr=rnd(B, L, D).to(DT[res]), dh=rnd(B, L, D).to(DT[blk]))
    if post == "none":
        t["post_weight"] = None
    return t


def _n(t):
    return None if t is None else t.double().numpy()


def _close(got, ref, terms, rel, dtype, what):
    bound = rel * terms + (2.0 ** -8 * np.abs(ref) if dtype == torch.bfloat16
                           else 0) + 1e-30
    err = np.abs(got.cpu().double().numpy() - ref)
    assert err.shape == ref.shape
    assert (err <= bound).all(), (what, float((err / bound).max()))


def _fwd_terms(t, pre, post, a, eps):
    """|a x| + |gate| |u|, and the h formula's absolute terms."""
    L = t["x"].shape[1]
    x, y = _n(t["x"]), _n(t["y"])
    u = 0.0
    if y is not None:
        _, ry = BN.unit(y, post, eps)
        mu = y.mean(-1, keepdims=True) if post == "layer" else 0.0
        pw = 1.0 if t["post_weight"] is None else np.abs(_n(t["post_weight"]))
        u = np.abs(BN.per_token(_n(t["gate"]), L, 1.0)) * pw * ry * (
            np.abs(y) + np.abs(mu))
    rt = abs(a) * np.abs(x) + u
    r, _ = BN.forward(x, y, _n(t["gate"]), None, None, None,
                      _n(t["post_weight"]), pre, post, eps, a)
    _, rho = BN.unit(r, pre, eps)
    mu = r.mean(-1, keepdims=True) if pre == "layer" else 0.0
    ht = rho * (rt + np.abs(mu) + np.abs(r))
    if t["pre_weight"] is not None:
        ht = ht * np.abs(_n(t["pre_weight"]))
    ht = ht * (1 + np.abs(BN.per_token(_n(t["scale"]), L, 0.0))) + np.abs(
        BN.per_token(_n(t["shift"]), L, 0.0))
    return rt, ht


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("absent", [(), ("gate", "shift"), ("scale",),
                                    ("pre_weight", "post_weight"), ("y",)])
def test_forward(case, absent):
    from paper_2609_36757_gb300 import fastvr as FV
    c = CASES[case]
    pre, post = c[4], c[5]
    t = _make(c, case)
    for name in absent:
        t[name] = None
    names = ("gate", "scale", "shift", "pre_weight", "post_weight")
    kw = {n: t[n] for n in names}
    a, eps = 0.75, 1e-5
    cfg = FV.make_norm_config(pre, post, eps=eps, residual_scale=a)
    dev = lambda v: None if v is None else v.cuda()
    dkw = {n: dev(v) for n, v in kw.items()}
    x, y = t["x"].cuda(), dev(t["y"])
    blk = DT[c[7]]
    r, h = FV.gated_norm(cfg, x, y, **dkw, block_dtype=blk)
    ref_r, ref_h = BN.forward(_n(t["x"]), _n(t["y"]),
                              *(_n(kw[n]) for n in names), pre, post, eps, a)
    rt, ht = _fwd_terms(t, pre, post, a, eps)
    _close(r, ref_r, rt, 1e-5, t["x"].dtype, "r")
    assert h.dtype == blk
    _close(h, ref_h, ht, 1e-5, blk, "h")
    # one output at a time, and in place
    assert torch.equal(FV.gated_norm(cfg, x, y, **dkw, block_dtype=blk,
                                     want_r=False)[1], h)
    assert torch.equal(FV.gated_norm(cfg, x, y, **dkw, want_h=False)[0], r)


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("absent", [(), ("dr",), ("dh",), ("y",),
                                    ("gate", "pre_weight"),
                                    ("scale", "post_weight")])
def test_backward(case, absent):
    from paper_2609_36757_gb300 import fastvr as FV
    c = CASES[case]
    B, G, T, D, pre, post = c[:6]
    t = _make(c, 50 + case)
    for name in absent:
        t[name] = None
    a, eps = 1.5, 1e-5
    cfg = FV.make_norm_config(pre, post, eps=eps, residual_scale=a)
    dev = {n: (None if v is None else v.cuda()) for n, v in t.items()}
    args = (dev["dr"], dev["dh"], dev["x"], dev["y"])
    kw = {n: dev[n] for n in ("gate", "scale", "pre_weight", "post_weight")}
    got = FV.gated_norm_bwd(cfg, *args, **kw, want_dshift=True)
    ref = BN.backward(_n(t["dr"]), _n(t["dh"]), _n(t["x"]), _n(t["y"]),
                      _n(t["gate"]), _n(t["scale"]), _n(t["pre_weight"]),
                      _n(t["post_weight"]), pre, post, eps, a, groups=G)
    # absolute terms of dx and dy
    L = G * T
    r, zero = _n(t["x"]), np.zeros((B, L, D))
    dh = zero if t["dh"] is None else _n(t["dh"])
    n, rho = BN.unit(r, pre, eps)
    mu = r.mean(-1, keepdims=True) if pre == "layer" else 0.0
    na = rho * (np.abs(r) + np.abs(mu))  # n with its cancellation
    w = 1.0 if t["pre_weight"] is None else np.abs(_n(t["pre_weight"]))
    dn = np.abs(dh) * (1 + np.abs(BN.per_token(_n(t["scale"]), L, 0.0))) * w
    avg = lambda v: v.mean(-1, keepdims=True)
    terms = (0 if t["dr"] is None else np.abs(_n(t["dr"]))) + rho * (
        dn + avg(dn) + na * avg(dn * na))
    _close(got.dx, ref["dx"], a * terms, 1e-5, t["x"].dtype, "dx")
    if t["y"] is not None:
        y = _n(t["y"])
        pw = 1.0 if t["post_weight"] is None else np.abs(_n(t["post_weight"]))
        du = terms * np.abs(BN.per_token(_n(t["gate"]), L, 1.0)) * pw
        yt = du
        ya = np.abs(y)
        if post != "none":
            _, ry = BN.unit(y, post, eps)
            mu = y.mean(-1, keepdims=True) if post == "layer" else 0.0
            ya = ry * (np.abs(y) + np.abs(mu))
            yt = ry * (du + avg(du) + ya * avg(du * ya))
        _close(got.dy, ref["dy"], yt, 1e-5, t["y"].dtype, "dy")
        fold = lambda v: v.reshape(B, G, T, D).sum(2)
        if got.dgate is not None:
            _close(got.dgate, ref["dgate"], fold(terms * ya * pw), 4e-5,
                   torch.float32, "dgate")
        if got.dpost_weight is not None:
            g = np.abs(BN.per_token(_n(t["gate"]), L, 1.0))
            _close(got.dpost_weight, ref["dpost_weight"],
                   (terms * g * ya).sum((0, 1)), 4e-5, torch.float32, "dpost")
    else:
        assert got.dy is None and got.dgate is None
    f32 = torch.float32
    fold = lambda v: v.reshape(B, G, T, D).sum(2)
    # without gate and scale the groups are one per batch entry
    if got.dscale is not None:
        _close(got.dscale, ref["dscale"], fold(np.abs(dh) * na * w), 4e-5, f32,
               "dscale")
    if got.dshift.shape[1] == G:
        _close(got.dshift, ref["dshift"], ref["dshift_abs"], 4e-5, f32,
               "dshift")
    if got.dpre_weight is not None:
        s1 = 1 + np.abs(BN.per_token(_n(t["scale"]), L, 0.0))
        _close(got.dpre_weight, ref["dpre_weight"],
               (np.abs(dh) * s1 * na).sum((0, 1)), 4e-5, f32, "dpre")
    again = FV.gated_norm_bwd(cfg, *args, **kw, want_dshift=True)
    for p, q in zip(got, again):
        assert (p is None and q is None) or torch.equal(p, q)


def test_in_place_and_other_stream():
    from paper_2609_36757_gb300 import fastvr as FV
    t = {n: v.cuda() for n, v in _make(CASES[6], 9).items()}
    cfg = FV.make_norm_config("rms", "rms")
    kw = {n: t[n] for n in ("gate", "scale", "shift", "pre_weight",
                            "post_weight")}
    r, h = FV.gated_norm(cfg, t["x"], t["y"], **kw)
    c = FV._norm_call(cfg, t["x"], (t["y"],), (), ())
    c.groups = 2
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x, h2 = t["x"].clone(), torch.empty_like(h)
    side.wait_stream(torch.cuda.current_stream())
    FV.fastvr_gated_norm_fwd(c, x.data_ptr(), t["y"].data_ptr(),
                             *(v.data_ptr() for v in kw.values()),
                             x.data_ptr(), h2.data_ptr(), side.cuda_stream)
    side.synchronize()
    assert torch.equal(x, r) and torch.equal(h2, h)


def test_bad_tensors():
    from paper_2609_36757_gb300 import fastvr as FV
    t = {n: (None if v is None else v.cuda())
         for n, v in _make(CASES[2], 9).items()}
    cfg = FV.make_norm_config("layer", "layer")
    ok = dict(x=t["x"], y=t["y"], gate=t["gate"], scale=t["scale"],
              pre_weight=t["pre_weight"])
    FV.gated_norm(cfg, **ok)
    for bad in (dict(x=t["x"][0]), dict(x=t["x"].half()),
                dict(x=t["x"].cpu()), dict(x=t["x"].transpose(0, 1)),
                dict(y=t["y"][:, :6]), dict(y=t["y"].half()),
                dict(gate=t["gate"].double()), dict(gate=t["gate"][:, :1]),
                dict(gate=t["gate"][:1]), dict(scale=t["scale"][..., :8]),
                dict(pre_weight=t["pre_weight"][:8]),
                dict(pre_weight=t["pre_weight"].bfloat16())):
        with pytest.raises(ValueError):
            FV.gated_norm(cfg, **{**ok, **bad})
    with pytest.raises(FV.FastVRError):  # 15 tokens in 2 groups
        FV.gated_norm(cfg, t["x"], t["y"],
                      gate=t["gate"][:, :2].contiguous())
