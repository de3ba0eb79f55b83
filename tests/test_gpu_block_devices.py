"""Tensors in host memory are refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_attention_outputs_in_host_memory():
    from paper_2609_36757_gb300 import fastvr as FV
    att = FV.StreamingAttention4(FV.make_config(1, 2, 64, 1, 1, 3))
    t = torch.ones(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    att.append(t, t)
    ref, lse = att.forward(t, want_lse=True)
    count = att.launch_count()
    for kw in (dict(out=torch.empty_like(ref, device="cpu")),
               dict(lse=torch.empty_like(lse, device="cpu")),
               dict(first_chunk=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            att.forward(t, **kw)
    for k, v in ((t.cpu(), t), (t, t.cpu())):
        with pytest.raises(ValueError):
            att.append(k, v)
    assert att.launch_count() == count and att.state() == (1, 1)
    out, l2 = torch.empty_like(ref), torch.empty_like(lse)
    att.forward(t, out=out, lse=l2)
    assert torch.equal(out, ref) and torch.equal(l2, lse)


def test_gradients_in_host_memory():
    from paper_2609_36757_gb300 import fastvr as FV
    g = torch.Generator("cuda").manual_seed(1)
    rnd = lambda: torch.randn(1, 4, 64, generator=g,
                              device="cuda").to(torch.bfloat16)
    a = dict(dr=rnd(), dh=rnd(), r=rnd(), y=rnd())
    cfg = FV.make_norm_config("layer", "rms")
    FV.gated_norm_bwd(cfg, **a)
    for name in a:
        with pytest.raises(ValueError):
            FV.gated_norm_bwd(cfg, **{**a, name: a[name].cpu()})
