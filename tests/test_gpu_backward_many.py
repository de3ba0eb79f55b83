"""The one-shot backward many times over: its compute warps go at their own
pace, and every call gives the first one's bits with no wait run out."""
import pytest
import torch

from paper_2609_36757_gb300 import workloads as WL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head_dim", [64, 128])
def test_backward_many_times(head_dim):
    from paper_2609_36757_gb300 import fastvr as FV
    w = WL.custom("many", batch=1, heads=6, head_dim=head_dim,
                  tokens_per_frame=300, frames_per_chunk=2, num_chunks=3,
                  window_chunks=1, seed=43)
    q, k, v = (torch.cat(t, 1).cuda() for t in
               zip(*(c[1:] for c in WL.chunk_stream(w))))
    cfg = FV.config_from_workload(w)
    out, lse = FV.blockcausal_attention(cfg, q, k, v, want_lse=True)
    do = torch.randn_like(q.float()).to(torch.bfloat16)
    first = FV.blockcausal_attention_bwd(cfg, q, k, v, out, do, lse)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(1000):
        for a, b in zip(FV.blockcausal_attention_bwd(cfg, q, k, v, out, do,
                                                     lse), first):
            differ += (a != b).sum()
    assert int(differ) == 0
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
