"""The block of examples/conditioned_block.py, its operators together: training
step against autograd in float64, single tokens against the same tokens of a
longer call."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import conditioned_block
    finally:
        sys.path.pop(0)
    return conditioned_block


def rel(a, b):
    a, b = a.detach().double().cpu(), b.detach().double().cpu()
    return float((a - b).norm() / b.norm())


def _reference(block, x, states, dr, lens, kind):
    """The block in float64 on the CPU, by autograd."""
    leaf = {n: getattr(block, n) for n in block.WEIGHTS}
    leaf.update(block.mod, x=x, states=states)
    t = {n: a.detach().double().cpu().requires_grad_()
         for n, a in leaf.items()}
    f = torch.nn.functional
    norm = lambda a: f.layer_norm(a, a.shape[-1:], eps=1e-6)
    B, L, D = x.shape
    K, d = block.kv_heads, block.d
    n1 = norm(t["x"]) * (1 + t["scale"]) + t["shift"]
    q = (n1 @ t["w_q"].T).view(B, L, K, -1, d)
    kv = (t["states"] @ t["w_kv"].T).view(B, -1, 2 * K, d)
    rows = []
    for b in range(B):
        n = kv.shape[1] if lens is None else lens[b]
        if n == 0:
            rows.append(torch.zeros(L, D, dtype=torch.float64))
            continue
        s = torch.einsum("lkgd,tkd->kglt", q[b], kv[b, :n, :K]) * d ** -0.5
        rows.append(torch.einsum("kglt,tkd->lkgd", s.softmax(-1),
                                 kv[b, :n, K:]).reshape(L, D))
    y1 = torch.stack(rows) @ t["w_o"].T
    r1 = t["x"] + t["gate"] * y1
    n2 = norm(r1) * (1 + t["scale2"]) + t["shift2"]
    act = f.silu if kind == "silu" else lambda a: f.gelu(
        a, approximate="tanh" if kind == "gelu_tanh" else "none")
    h = act(n2 @ t["w_gate"].T) * (n2 @ t["w_up"].T)
    r2 = r1 + t["gate2"] * (h @ t["w_down"].T)
    names = list(t)
    grads = torch.autograd.grad(r2, [t[n] for n in names],
                                dr.double().cpu(), allow_unused=True)
    return r2, dict(zip(names, grads))


@pytest.mark.parametrize("B,L,T,heads,kv_heads,d,lens,kind", [
    (1, 300, 70, 4, 4, 64, None, "silu"),
    (2, 150, 200, 4, 2, 128, [200, 33], "gelu_tanh"),
    (3, 20, 40, 2, 1, 64, [40, 0, 9], "gelu"),
    (1, 1, 30, 4, 2, 64, None, "silu"),
])
def test_training_step(ex, B, L, T, heads, kv_heads, d, lens, kind):
    """On the longest way a value passes about twelve bfloat16 roundings
    (activations, projections, products' operands and results), each of relative
    size 2^-8 at most and 2^-8 / sqrt(3) on average over a tensor; their sum as
    if all agreed is 12 x 2^-8 / sqrt(3) = 2.7e-2."""
    block = ex.Conditioned(heads, kv_heads, 96, 200, B, 5, d, kind)
    g = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(*s, generator=g,
                                 device="cuda").to(torch.bfloat16)
    x, states, dr = rnd(B, L, block.dim), rnd(B, T, 96), rnd(B, L, block.dim)
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32,
                                                    device="cuda")
    r, grads = ex.train_step(block, x, states, dr, kv_len)
    assert ex.FV.fastvr_get_device_status() == ex.FV.FASTVR_OK
    ref, want = _reference(block, x, states, dr, lens, kind)
    assert rel(r, ref) <= 2.7e-2
    assert set(grads) == set(want)
    for name, a in grads.items():
        assert rel(a, want[name]) <= 2.7e-2, name
    if lens is not None:
        for b, n in enumerate(lens):
            assert bool((grads["states"][b, n:] == 0).all())


def test_single_tokens_agree_with_a_chunk(ex):
    block = ex.Conditioned(4, 2, 96, 200, 2, 7, 64)
    g = torch.Generator(device="cuda").manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=g,
                                 device="cuda").to(torch.bfloat16)
    x, states = rnd(2, 70, block.dim), rnd(2, 90, 96)
    kv_len = torch.tensor([90, 17], dtype=torch.int32, device="cuda")
    k, v = block.prompt(states)
    whole = block.forward(x, k, v, kv_len)
    for i in (0, 31, 69):
        one = block.forward(x[:, i:i + 1].contiguous(), k, v, kv_len)
        # eight roundings on the way, of both
        assert rel(one[:, 0], whole[:, i]) <= 2 * 8 * 2.0 ** -8 / 3 ** 0.5


def test_replayed_training_step(ex):
    block = ex.Conditioned(4, 4, 96, 200, 1, 9, 64)
    g = torch.Generator(device="cuda").manual_seed(10)
    rnd = lambda *s: torch.randn(*s, generator=g,
                                 device="cuda").to(torch.bfloat16)
    x, states, dr = rnd(1, 260, 256), rnd(1, 140, 96), rnd(1, 260, 256)
    ex.train_step(block, x, states, dr)  # warm-up (library products)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, grads = ex.train_step(block, x, states, dr)
    x.copy_(rnd(1, 260, 256))
    graph.replay()
    r2, want = ex.train_step(block, x, states, dr)
    assert torch.equal(r, r2)
    for name in grads:
        assert torch.equal(grads[name], want[name]), name
