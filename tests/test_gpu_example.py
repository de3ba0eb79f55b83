"""The block of examples/streaming_block.py, all operators together: its
stream over the 4-bit cache against the bfloat16 cache, and its training step
against autograd in float64."""
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
        import streaming_block
    finally:
        sys.path.pop(0)
    return streaming_block


def rel(a, b):
    a, b = a.detach().double().cpu(), b.detach().double().cpu()
    return float((a - b).norm() / b.norm())


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (4, 2)])
def test_stream_over_both_caches(ex, heads, kv_heads):
    """A 4-bit value is off by about 0.1 deviations (step max / 7 of 32 values,
    uniform rounding), in the scores and in the values: sqrt(2) 0.1 of the
    attention's output.  The post norm keeps that ratio, the residual (of the
    same size as the gated update or larger) lowers it."""
    block = ex.Block(heads, kv_heads, 6, 17)
    cfg = ex.attention_config(block, 2, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    xs = [torch.randn(1, 2 * block.frame, block.dim, generator=g,
                      device="cuda").to(torch.bfloat16) for _ in range(5)]
    ref, _ = ex.stream(block, ex.FV.StreamingAttention(cfg), xs, 2)
    got, _ = ex.stream(block, ex.FV.StreamingAttention4(cfg, kv_heads), xs, 2)
    for (r0, h0), (r1, h1), x in zip(ref, got, xs):
        assert rel(r1, r0) <= 0.14
        assert rel(h1, h0) <= 0.14
        assert rel(r0, x) > 0.05  # the update is there at all


def _reference(ex, block, x, dr, dh, k, window):
    """The block in float64 on the CPU, by autograd."""
    P = {n: t.detach().double().cpu().requires_grad_()
         for n, t in dict(x=x, w_qkv=block.w_qkv, w_out=block.w_out,
                          post_weight=block.post_weight,
                          **block.mod).items()}
    B, L, D = x.shape
    H, d = block.heads, block.d

    def layer(v):
        return (v - v.mean(-1, keepdim=True)) / torch.sqrt(
            v.var(-1, unbiased=False, keepdim=True) + 1e-6)

    n = layer(P["x"]) * (1 + P["scale"]) + P["shift"]
    q, k_, v = (n @ P["w_qkv"].T).view(B, L, 3 * H, d).split(H, 2)
    theta, _ = ex.FV.fastvr_rotary_frequencies(block.rot)
    sections = list(block.rot.section)
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(sections))
    pos = block.positions(0, L // block.frame).cpu().double()
    ang = (pos[:, axis] * torch.tensor(theta, dtype=torch.float64))[None, :, None]

    def rotate(t):
        a, b = t[..., 0::2], t[..., 1::2]
        return torch.stack([a * ang.cos() - b * ang.sin(),
                            b * ang.cos() + a * ang.sin()], -1).flatten(-2)

    chunk = torch.arange(L) // (k * block.frame)
    gap = chunk[:, None] - chunk[None]
    s = torch.einsum("blhd,bmhd->bhlm", rotate(q), rotate(k_)) * d ** -0.5
    s = s.masked_fill((gap < 0) | (gap > window), -torch.inf)
    o = torch.einsum("bhlm,bmhd->blhd", s.softmax(-1), v).reshape(B, L, D)
    y = o @ P["w_out"].T
    u = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * P["post_weight"]
    r = P["x"] + P["gate"] * u
    h = layer(r) * (1 + P["scale2"]) + P["shift2"]
    ((r * dr.double().cpu()).sum() + (h * dh.double().cpu()).sum()).backward()
    return r, h, {n: t.grad for n, t in P.items()}


def test_train_step_matches_autograd(ex):
    """About fifteen tensors between the input and a gradient are rounded to
    bfloat16 (2^-9 each, relative): 15 2^-9 = 0.03."""
    block = ex.Block(2, 2, 5, 7)
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda: torch.randn(1, 6 * block.frame, block.dim, generator=g,
                              device="cuda").to(torch.bfloat16)
    x, dr, dh = rnd(), rnd(), rnd()
    r, h, grads = ex.train_step(block, x, dr, dh, 2, 1)
    rr, rh, rg = _reference(ex, block, x, dr, dh, 2, 1)
    assert rel(r, rr) <= 0.03 and rel(h, rh) <= 0.03
    assert set(grads) == set(rg)
    for name in sorted(grads):
        got = grads[name].double().cpu().reshape(rg[name].shape)
        assert rel(got, rg[name]) <= 0.03, name


def test_command(ex, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["streaming_block.py", "--chunks", "3",
                                      "--heads", "2", "--rows", "4", "--cols",
                                      "9"])
    ex.main()
    out = capsys.readouterr().out
    assert "4-bit" in out and "differ by" in out
