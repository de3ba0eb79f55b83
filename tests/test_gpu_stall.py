"""The streamed and the one-shot forward without their values, the one-shot backward
without its second step's tiles: waits run out while the MMA warp is amid its work, the
forward's softmax lanes' each at its own time.  The failure is reported, every role
leaves soon, and the same call gives its results again."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


def _rnd(seed, *shape):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def _streamed(chunks, n, heads, d, window):
    from paper_2609_36757_gb300 import fastvr as FV
    att = FV.StreamingAttention(FV.make_config(1, heads, d, n, 1, window,
                                               chunks))
    for c in range(chunks):
        att.append(_rnd(c, 1, n, heads, d), _rnd(500 + c, 1, n, heads, d))
    q = _rnd(1000, 1, n, heads, d)
    return (lambda: att.forward(q, want_lse=True), att.status,
            lambda *a: FV.fastvr_debug_inject_stall(att.plan, *a))


def _one_shot(chunks, n, heads, d, window):
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_config(1, heads, d, n, 1, window, chunks)
    q, k, v = (_rnd(i, 1, chunks * n, heads, d) for i in range(3))
    return (lambda: FV.blockcausal_attention(cfg, q, k, v, want_lse=True),
            FV.fastvr_get_device_status, FV.fastvr_debug_inject_stall_noplan)


def _backward(chunks, n, heads, d, window):
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_config(1, heads, d, n, 1, window, chunks)
    q, k, v, do = (_rnd(i, 1, chunks * n, heads, d) for i in range(4))
    out, lse = FV.blockcausal_attention(cfg, q, k, v, want_lse=True)
    return (lambda: FV.blockcausal_attention_bwd(cfg, q, k, v, out, do, lse),
            FV.fastvr_get_device_status, FV.fastvr_debug_inject_stall_noplan)


@pytest.mark.parametrize("case", [
    # chunks, tokens of each, heads, window: whole units; units cut over CTAs and
    # merged; units of several hundred key tiles
    (3, 700, 2, -1), (2, 5000, 40, 1), (80, 200, 1, -1), (300, 200, 2, -1),
    (4, 20000, 1, -1)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [_streamed, _one_shot, _backward])
def test_stall_amid_a_unit_is_reported(make, d, case):
    from paper_2609_36757_gb300 import fastvr as FV
    chunks, n, heads, window = case
    call, status, stall = make(chunks, n, heads, d, window)
    ref = call()
    assert status() == FV.FASTVR_OK
    for limit in (1_000_000, 20_000_000):  # 1 and 20 ms per wait
        stall(2, limit)
        try:
            t0 = time.perf_counter()
            call()
            got = status()
            assert time.perf_counter() - t0 < 2.0
        finally:
            stall(0, 0)
        assert got == FV.FASTVR_ERR_TIMEOUT
        assert status() == FV.FASTVR_OK  # cleared
    for a, b in zip(call(), ref):
        assert torch.equal(a, b)
    assert status() == FV.FASTVR_OK


@pytest.mark.parametrize("stall", [-1, 3, 1 << 20])
@pytest.mark.parametrize("make", [_streamed, _one_shot, _backward])
def test_any_other_value_stalls_the_mma_warp(make, stall):
    from paper_2609_36757_gb300 import fastvr as FV
    call, status, hook = make(3, 300, 2, 64, -1)
    call()
    hook(stall, 5_000_000)
    try:
        call()
        assert status() == FV.FASTVR_ERR_TIMEOUT
    finally:
        hook(0, 0)
    call()
    assert status() == FV.FASTVR_OK
