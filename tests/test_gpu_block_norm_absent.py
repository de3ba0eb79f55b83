"""The gated norm on the GPU with a weight that it does not use: no post norm,
but a post weight.  The outputs do not depend on it, so its gradient is zero,
exactly, and every other gradient is what it is without the weight, bit for
bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


# groups cut into slices, whole groups to a CTA, rows side by side
@pytest.mark.parametrize("batch,groups,tokens,dim", [
    (1, 2, 40, 1536), (2, 400, 1, 512), (3, 5, 7, 64), (1, 1, 1, 8192)])
@pytest.mark.parametrize("with_pre", [False, True])
def test_post_weight_without_a_post_norm(batch, groups, tokens, dim, with_pre):
    from paper_2609_36757_gb300 import fastvr as FV
    g = torch.Generator("cuda").manual_seed(dim)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    L = groups * tokens
    x, y, dr, dh = (rnd(batch, L, dim).to(torch.bfloat16) for _ in range(4))
    kw = dict(gate=rnd(batch, groups, dim), scale=rnd(batch, groups, dim),
              pre_weight=rnd(dim) if with_pre else None)
    cfg = FV.make_norm_config("layer", "none")
    w = rnd(dim)
    plain = FV.gated_norm(cfg, x, y, **kw)
    given = FV.gated_norm(cfg, x, y, **kw, post_weight=w)
    assert all(torch.equal(a, b) for a, b in zip(plain, given))
    ref = FV.gated_norm_bwd(cfg, dr, dh, plain[0], y, **kw)
    got = FV.gated_norm_bwd(cfg, dr, dh, plain[0], y, **kw, post_weight=w)
    assert ref.dpost_weight is None
    assert got.dpost_weight.shape == (dim,) and (got.dpost_weight == 0).all()
    for name in ("dx", "dy", "dgate", "dscale", "dshift", "dpre_weight"):
        a, b = getattr(ref, name), getattr(got, name)
        assert (a is None and b is None) or torch.equal(a, b), name
