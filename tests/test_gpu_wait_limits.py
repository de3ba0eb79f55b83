"""Wait limits outside the range that kernels can keep are brought into it: with the
shortest, calls that finish within a millisecond give their results, since no wait of
theirs, nor the last one for copies in flight, ends before."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _calls():
    from paper_2609_36757_gb300 import fastvr as FV
    g = torch.Generator("cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g,
                                 device="cuda").to(torch.bfloat16)
    q, k, v, do = (rnd(1, 400, 2, 64) for _ in range(4))
    x, wg, wu, dh = rnd(300, 200), rnd(136, 200), rnd(136, 200), rnd(300, 136)
    cc, fc = FV.make_cross_config(), FV.make_ffn_config()
    oc = FV.make_config(1, 2, 64, 200, 1, 1)

    def cross():
        out, lse = FV.cross_attention(cc, q, k, v, want_lse=True)
        return (out, lse) + tuple(
            FV.cross_attention_bwd(cc, q, k, v, out, do, lse))

    def ffn():
        h, saved = FV.gated_ffn(fc, x, wg, wu, want_saved=True)
        return (h,) + tuple(FV.gated_ffn_bwd(fc, dh, x, wg, wu, saved))

    def one_shot():
        out, lse = FV.blockcausal_attention(oc, q, k, v, want_lse=True)
        return (out, lse) + tuple(
            FV.blockcausal_attention_bwd(oc, q, k, v, out, do, lse))

    return dict(cross=cross, ffn=ffn, one_shot=one_shot)


@pytest.mark.parametrize("limit", [1, 1000, 2 ** 64 - 1])
@pytest.mark.parametrize("name", ["cross", "ffn", "one_shot"])
def test_calls_without_a_plan(name, limit):
    from paper_2609_36757_gb300 import fastvr as FV
    call = _calls()[name]
    ref = call()
    torch.cuda.synchronize()
    FV.fastvr_debug_inject_stall_noplan(0, limit)
    try:
        got = call()
        assert FV.fastvr_get_device_status() == FV.FASTVR_OK
    finally:
        FV.fastvr_debug_inject_stall_noplan(0, 0)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("limit", [1, 1000, 2 ** 64 - 1])
def test_streaming_plan(limit):
    from paper_2609_36757_gb300 import fastvr as FV
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v = (torch.randn(1, 200, 2, 64, generator=g, device="cuda").to(
        torch.bfloat16) for _ in range(3))
    att = FV.StreamingAttention(FV.make_config(1, 2, 64, 200, 1, 1))
    att.append(k, v)
    ref = att.forward(q, want_lse=True)
    torch.cuda.synchronize()
    FV.fastvr_debug_inject_stall(att.plan, 0, limit)
    got = att.forward(q, want_lse=True)
    assert att.status() == FV.FASTVR_OK
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
