"""The type of the gated norm's h without a block output: bfloat16 or float32;
any other is refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["float16", "float64", "int8", "uint8",
                                  "float8_e4m3fn", "int16", "bool"])
def test_block_dtype_refused(name):
    from paper_2609_36757_gb300 import fastvr as FV
    x = torch.ones(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    cfg = FV.make_norm_config("rms")
    for kw in ({}, dict(want_r=False), dict(want_h=False)):
        with pytest.raises(ValueError):
            FV.gated_norm(cfg, x, None, block_dtype=getattr(torch, name), **kw)


def test_block_dtype_served():
    from paper_2609_36757_gb300 import fastvr as FV
    x = torch.randn(1, 4, 64, device="cuda").to(torch.bfloat16)
    cfg = FV.make_norm_config("rms")
    h = {t: FV.gated_norm(cfg, x, None, block_dtype=t)[1]
         for t in (None, torch.bfloat16, torch.float32)}
    assert h[None].dtype == torch.bfloat16
    assert all(h[t].dtype == t for t in h if t is not None)
    assert torch.equal(h[None], h[torch.bfloat16])
    full = h[torch.float32]  # rounded once: 2^-9 of it
    assert ((h[None].float() - full).abs() <= 2.0 ** -8 * full.abs()).all()
    # with a block output its type is h's, whatever is given
    y = torch.randn(1, 4, 64, device="cuda")
    assert FV.gated_norm(cfg, x, y)[1].dtype == torch.float32
    assert FV.gated_norm(cfg, x, y, block_dtype=torch.bfloat16)[1].dtype == \
        torch.float32
