"""Cross attention's forward without its values, and its gradients without some tiles:
waits run out while the MMA warp is amid a unit, the forward's softmax lanes' each at
its own time.  The failure is reported, every role leaves, and the same call gives its
results again."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


def _call(B, L, H, T, d, lens, seed=1, grads=False):
    from paper_2609_36757_gb300 import fastvr as FV
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g,
                                 device="cuda").to(torch.bfloat16)
    q, k, v = rnd(B, L, H, d), rnd(B, T, 1, d), rnd(B, T, 1, d)
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32,
                                               device="cuda")
    cfg = FV.make_cross_config()
    if not grads:
        return lambda: FV.cross_attention(cfg, q, k, v, n, want_lse=True)
    out, lse = FV.cross_attention(cfg, q, k, v, n, want_lse=True)
    do = rnd(B, L, H, d)
    return lambda: FV.cross_attention_bwd(cfg, q, k, v, out, do, lse, n)


CASES = [
    # B, L, H, T, d, lens
    (1, 300, 2, 300, 128, None),
    (1, 300, 2, 300, 64, None),
    (3, 700, 4, 200, 128, [200, 0, 77]),
    (3, 700, 60, 140, 64, [140, 0, 77]),  # several units to a CTA
]


@pytest.mark.parametrize("grads", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_stall_amid_a_unit_is_reported(case, grads):
    from paper_2609_36757_gb300 import fastvr as FV
    call = _call(*case, grads=grads)
    ref = call()
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
    FV.fastvr_debug_inject_stall_noplan(2, 20_000_000)  # 20 ms per wait
    try:
        t0 = time.perf_counter()
        call()
        status = FV.fastvr_get_device_status()
        assert time.perf_counter() - t0 < 5.0
    finally:
        FV.fastvr_debug_inject_stall_noplan(0, 0)
    assert status == FV.FASTVR_ERR_TIMEOUT
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK  # cleared
    for a, b in zip(call(), ref):
        assert torch.equal(a, b)
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK


@pytest.mark.parametrize("grads", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_stall_amid_a_long_unit(d, grads):
    """The MMA warp leaves a unit of 1563 key tiles soon, whatever the limit: what
    keeps it from waiting for arrivals that nobody makes lasts for a while only."""
    from paper_2609_36757_gb300 import fastvr as FV
    call = _call(1, 300, 1, 200_000, d, None, grads=grads)
    ref = call()
    FV.fastvr_debug_inject_stall_noplan(2, 1_000_000)  # 1 ms
    try:
        t0 = time.perf_counter()
        call()
        status = FV.fastvr_get_device_status()
        assert time.perf_counter() - t0 < 0.5
    finally:
        FV.fastvr_debug_inject_stall_noplan(0, 0)
    assert status == FV.FASTVR_ERR_TIMEOUT
    for a, b in zip(call(), ref):
        assert torch.equal(a, b)
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
