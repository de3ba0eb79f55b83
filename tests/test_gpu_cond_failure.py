"""Cross attention and the gated feed-forward: bounded waits that run out are
reported and leave the context usable; first calls under capture; tensors in
host memory; calls from two threads; tensors past 2^31 elements."""
import os
import subprocess
import sys
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _rnd(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g,
                                  device="cuda").to(torch.bfloat16)


def _calls(FV, seed=1):
    """(name, call) of the tile kernels; a call returns its results."""
    rnd = _rnd(seed)
    q, k, v = rnd(2, 700, 4, 128), rnd(2, 300, 2, 128), rnd(2, 300, 2, 128)
    do = rnd(2, 700, 4, 128)
    lens = torch.tensor([300, 140], dtype=torch.int32, device="cuda")
    cc = FV.make_cross_config()
    out, lse = FV.cross_attention(cc, q, k, v, lens, want_lse=True)
    x, wg, wu, dh = rnd(600, 200), rnd(328, 200), rnd(328, 200), rnd(600, 328)
    fc = FV.make_ffn_config("silu")
    _, saved = FV.gated_ffn(fc, x, wg, wu, want_saved=True)
    return [
        ("cross", lambda: FV.cross_attention(cc, q, k, v, lens,
                                             want_lse=True)),
        ("cross_bwd", lambda: FV.cross_attention_bwd(cc, q, k, v, out, do,
                                                     lse, lens)),
        ("ffn", lambda: (FV.gated_ffn(fc, x, wg, wu),)),
        ("ffn_bwd", lambda: FV.gated_ffn_bwd(fc, dh, x, wg, wu, saved)),
    ]


@pytest.mark.parametrize("which", range(4))
def test_timeout_is_reported_and_context_survives(which):
    from paper_2609_36757_gb300 import fastvr as FV
    name, call = _calls(FV)[which]
    ref = call()
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
    FV.fastvr_debug_inject_stall_noplan(1, 20_000_000)  # 20 ms per wait
    try:
        t0 = time.perf_counter()
        call()
        status = FV.fastvr_get_device_status()
        assert time.perf_counter() - t0 < 5.0
    finally:
        FV.fastvr_debug_inject_stall_noplan(0, 0)
    assert status == FV.FASTVR_ERR_TIMEOUT, name
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK  # cleared
    for a, b in zip(call(), ref):
        assert torch.equal(a, b)
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK


FIRST = """
import sys
import torch
sys.path.insert(0, {root!r})
from paper_2609_36757_gb300 import fastvr as FV
g = torch.Generator(device="cuda").manual_seed(1)
rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
L = {tokens}
q, k, v, do = rnd(1, L, 2, 64), rnd(1, 150, 2, 64), rnd(1, 150, 2, 64), \
    rnd(1, L, 2, 64)
x, wg, wu, dh = rnd(L, 64), rnd(72, 64), rnd(72, 64), rnd(L, 72)
cc, fc = FV.make_cross_config(), FV.make_ffn_config()
def run():
    out, lse = FV.cross_attention(cc, q, k, v, want_lse=True)
    h, saved = FV.gated_ffn(fc, x, wg, wu, want_saved=True)
    return (out, lse, h) + tuple(FV.cross_attention_bwd(
        cc, q, k, v, out, do, lse)) + tuple(FV.gated_ffn_bwd(
            fc, dh, x, wg, wu, saved))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    held = run()
graph.replay()
torch.cuda.synchronize()
for a, b in zip(held, run()):
    assert torch.equal(a, b)
print("same")
"""


@pytest.mark.parametrize("tokens", [1, 300])
def test_first_calls_of_a_process_may_be_captured(tokens):
    r = subprocess.run(
        [sys.executable, "-c", FIRST.format(root=ROOT, tokens=tokens)],
        capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_host_tensors_are_refused():
    from paper_2609_36757_gb300 import fastvr as FV
    rnd = _rnd(2)
    c = dict(q=rnd(1, 3, 2, 64), k=rnd(1, 5, 2, 64), v=rnd(1, 5, 2, 64),
             kv_len=torch.tensor([4], dtype=torch.int32, device="cuda"))
    cfg = FV.make_cross_config()
    out, lse = FV.cross_attention(cfg, **c, want_lse=True)
    b = dict(c, out=out, dout=out.clone(), lse=lse)
    for name in c:
        with pytest.raises(ValueError):
            FV.cross_attention(cfg, **{**c, name: c[name].cpu()})
    for name in b:
        with pytest.raises(ValueError):
            FV.cross_attention_bwd(cfg, **{**b, name: b[name].cpu()})
    f = dict(x=rnd(3, 64), w_gate=rnd(8, 64), w_up=rnd(8, 64))
    cfg = FV.make_ffn_config()
    h, saved = FV.gated_ffn(cfg, **f, want_saved=True)
    for name in f:
        with pytest.raises(ValueError):
            FV.gated_ffn(cfg, **{**f, name: f[name].cpu()})
        with pytest.raises(ValueError):
            FV.gated_ffn_bwd(cfg, h, saved=saved, **{**f, name: f[name].cpu()})
    for dh, s in ((h.cpu(), saved), (h, (saved[0].cpu(), saved[1])),
                  (h, (saved[0], saved[1].cpu()))):
        with pytest.raises(ValueError):
            FV.gated_ffn_bwd(cfg, dh, saved=s, **f)


def test_two_threads_on_their_own_streams():
    from paper_2609_36757_gb300 import fastvr as FV
    calls = [_calls(FV, s) for s in (3, 4)]
    want = [[c() for _, c in cs] for cs in calls]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                for (name, c), ref in zip(calls[i], want[i]):
                    for a, b in zip(c(), ref):
                        if not torch.equal(a, b):
                            wrong.append((i, name))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK


def test_cross_past_31_bits():
    """2.3e9 elements of q: rows at the far end equal a call on them alone."""
    from paper_2609_36757_gb300 import fastvr as FV
    rnd = _rnd(5)
    L, H, d, T = 1_130_000, 16, 128, 40
    q = torch.empty((1, L, H, d), dtype=torch.bfloat16, device="cuda")
    q.normal_(generator=torch.Generator(device="cuda").manual_seed(6))
    assert q.numel() > 2 ** 31
    k, v = rnd(1, T, 4, d), rnd(1, T, 4, d)
    cfg = FV.make_cross_config()
    out, lse = FV.cross_attention(cfg, q, k, v, want_lse=True)
    do = q  # any values serve
    grads = FV.cross_attention_bwd(cfg, q, k, v, out, do, lse)
    n = L - 4 * 128 * (L // (4 * 128)) + 512
    tail = q[:, L - n:]
    o2, l2 = FV.cross_attention(cfg, tail, k, v, want_lse=True)
    assert torch.equal(out[:, L - n:], o2)
    assert torch.equal(lse[..., L - n:], l2)
    g2 = FV.cross_attention_bwd(cfg, tail, k, v, o2, do[:, L - n:], l2)
    assert torch.equal(grads.dq[:, L - n:], g2.dq)
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK


def test_ffn_past_31_bits():
    """2.2e9 elements of h: rows at the far end equal a call on them alone."""
    from paper_2609_36757_gb300 import fastvr as FV
    rnd = _rnd(7)
    M, D, F = 1_100_000, 64, 2048
    x, wg, wu = rnd(M, D), rnd(F, D), rnd(F, D)
    cfg = FV.make_ffn_config("gelu_tanh")
    h, saved = FV.gated_ffn(cfg, x, wg, wu, want_saved=True)
    assert h.numel() > 2 ** 31
    g = FV.gated_ffn_bwd(cfg, h, x, wg, wu, saved)
    n = 1000
    h2, s2 = FV.gated_ffn(cfg, x[-n:], wg, wu, want_saved=True)
    assert torch.equal(h[-n:], h2)
    for a, b in zip(saved, s2):
        assert torch.equal(a[-n:], b)
    g2 = FV.gated_ffn_bwd(cfg, h2, x[-n:], wg, wu, s2)
    assert torch.equal(g.dx[-n:], g2.dx)
    # the weights' sums run over all rows in float32; in pieces they differ by
    # rounding only: M u of the absolute terms would be far more
    part = sum(FV.gated_ffn_bwd(
        cfg, h[i:i + M // 4], x[i:i + M // 4], wg, wu,
        tuple(t[i:i + M // 4] for t in saved)).dw_gate.double()
        for i in range(0, M, M // 4))
    err = (g.dw_gate.double() - part).norm() / part.norm()
    assert float(err) <= 2.0 ** -7  # roundings of five bfloat16 results
    assert FV.fastvr_get_device_status() == FV.FASTVR_OK
