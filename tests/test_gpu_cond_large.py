"""Gradients that sum over more than 2^31 elements: all rows but the last ones have no
gradient of their own, so that the sums are the last rows' exactly, and the float64
oracle needs these only."""
import pytest
import torch

import test_gpu_cross as TC
import test_gpu_ffn as TF

pytestmark = pytest.mark.gpu

TAIL = 700


def test_cross_dk_dv_past_31_bits():
    from paper_2609_36757_gb300 import fastvr as FV
    L, H, d, T, K = 1_130_000, 16, 128, 40, 4
    g = torch.Generator(device="cuda").manual_seed(6)
    q, do = (torch.empty((1, L, H, d), dtype=torch.bfloat16, device="cuda")
             for _ in range(2))
    assert (L - TAIL) * H * d > 2 ** 31
    q.normal_(generator=g)
    do.zero_()
    do[:, L - TAIL:].normal_(generator=g)
    k, v = (torch.randn(1, T, K, d, generator=g, device="cuda").to(
        torch.bfloat16) for _ in range(2))
    cfg = FV.make_cross_config()
    out, lse = FV.cross_attention(cfg, q, k, v, want_lse=True)
    got = FV.cross_attention_bwd(cfg, q, k, v, out, do, lse)
    ref = TC.bounds(q[:, L - TAIL:], k, v, do[:, L - TAIL:], None, d ** -0.5)
    TC.close(got.dq[:, L - TAIL:], *ref[2], "dq")
    TC.close(got.dk, *ref[3], "dk")
    TC.close(got.dv, *ref[4], "dv")
    assert not bool(got.dq[:, :L - TAIL].any())
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK


@pytest.mark.parametrize("want_dw", [True, False])
def test_ffn_gradients_past_31_bits(want_dw):
    from paper_2609_36757_gb300 import fastvr as FV
    M, D, F = 1_100_000, 72, 2048
    assert (M - TAIL) * F > 2 ** 31
    x, wg, wu, dh = (t.cuda() for t in TF.make((TAIL, D, F, "silu"), 7))
    big = torch.empty((M, D), dtype=torch.bfloat16, device="cuda")
    big.normal_(generator=torch.Generator(device="cuda").manual_seed(8))
    big[-TAIL:] = x
    cfg = FV.make_ffn_config("silu")
    _, saved = FV.gated_ffn(cfg, big, wg, wu, want_saved=True)
    dhb = torch.zeros((M, F), dtype=torch.bfloat16, device="cuda")
    dhb[-TAIL:] = dh
    got = FV.gated_ffn_bwd(cfg, dhb, big, wg, wu, saved, want_dw=want_dw)
    ref = TF.bounds(x, wg, wu, dh, "silu")
    TF.close(got.dx[-TAIL:], *ref[3], "dx")
    assert not bool(got.dx[:-TAIL].any())
    if want_dw:
        TF.close(got.dw_gate, *ref[4], "dw_gate")
        TF.close(got.dw_up, *ref[5], "dw_up")
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
