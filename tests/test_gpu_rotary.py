"""Rotary positions on the GPU against the float64 oracle.

Bound of one element's error, from the kernel's arithmetic: the angle reaches
sincospi as a turn rounded to 2^-32 and to 24 bits of float (6e-8 of pi), the
frequency is held to 2^-53 (below that for |p| <= 2^24), sine and cosine add 2
units in the last place, the products and their sum 2 more: less than 1e-6
(|a| + |b|) m, and one rounding of the result to its type (2^-8 of it covers
bfloat16's half unit)."""
import numpy as np
import pytest
import torch

from oracle import rotary as OR

pytestmark = pytest.mark.gpu


def _inputs(B, L, H, Hk, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(B, L, H + 2 * Hk, d, generator=g).to(dtype)


def _partner(x, n, layout):
    """|a| + |b| of each element's pair."""
    m = np.abs(x)
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + n)
    s = m[..., a] + m[..., b]
    m[..., a] = m[..., b] = s
    return m


def _check(got, x, pos, cfgkw, dtype, transpose):
    sections = cfgkw.get("sections") or [cfgkw["rotary_dim"] // 2]
    theta, mag = OR.frequencies(
        sections, scaling=cfgkw.get("scaling", "none"),
        factors=cfgkw.get("factors"), contexts=cfgkw.get("original_contexts"))
    layout = cfgkw.get("layout", "interleaved")
    x = x.double().numpy()
    ref = OR.rotate(x, pos.numpy(), sections, theta, mag, layout, transpose)
    bound = 1e-6 * mag * _partner(x.copy(), len(theta), layout)
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * np.abs(ref)
    err = np.abs(got.cpu().double().numpy() - ref)
    assert (err <= bound).all(), float((err / bound).max())
    rot = 2 * len(theta)
    assert np.array_equal(got.cpu().double().numpy()[..., rot:], x[..., rot:])


CASES = [
    # B, L, H, Hk, d, config
    (1, 1, 1, 1, 64, dict(rotary_dim=64)),
    (1, 1, 1, 1, 8, dict(rotary_dim=2)),
    (3, 1, 8, 2, 128, dict(rotary_dim=128, layout="half", scaling="yarn",
                           factors=[8.0], original_contexts=[4096])),
    (2, 37, 4, 4, 128, dict(rotary_dim=128, sections=[22, 21, 21])),
    (2, 5, 3, 1, 128, dict(rotary_dim=104, layout="half", scaling="ntk",
                           factors=[4.0])),
    (1, 300, 12, 12, 64, dict(rotary_dim=40, layout="half", scaling="linear",
                              factors=[2.0])),
    (1, 33, 2, 1, 72, dict(rotary_dim=36, layout="half")),    # 18 pairs
    (1, 33, 2, 1, 72, dict(rotary_dim=30, layout="half")),    # 15 pairs
    (1, 70, 2, 2, 72, dict(rotary_dim=34)),   # ends inside a 16-byte piece
    (1, 9, 2, 2, 512, dict(rotary_dim=512, layout="half")),
    (1, 2500, 12, 12, 128, dict(rotary_dim=64, layout="half",
                                sections=[12, 10, 10])),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("transpose", [False, True])
def test_matches_the_definition(case, dtype, transpose):
    from paper_2609_36757_gb300 import fastvr as FV
    B, L, H, Hk, d, kw = CASES[case]
    cfg = FV.make_rotary_config(d, **kw)
    x = _inputs(B, L, H, Hk, d, dtype, 100 + case)
    g = torch.Generator().manual_seed(case)
    top = 1 << 20
    pos = torch.randint(-top, top, (B, L, cfg.axes), generator=g,
                        dtype=torch.int32)
    xd = x.cuda()   # q and k are slices of the fused projection: strided
    q, k = xd[:, :, :H], xd[:, :, H:H + Hk]
    f = FV.rotary_bwd if transpose else FV.rotary
    qo, ko = f(cfg, q, k, pos.cuda())
    _check(qo, x[:, :, :H], pos, kw, dtype, transpose)
    _check(ko, x[:, :, H:H + Hk], pos, kw, dtype, transpose)
    # shared positions, in place, q alone: bit for bit the same rows
    f(cfg, q, k, pos[:1].cuda(), out=(q, k))
    assert torch.equal(q[0].cpu(), qo[0].cpu())
    assert torch.equal(k[0].cpu(), ko[0].cpu())
    assert torch.equal(xd[:, :, H + Hk:].cpu(), x[:, :, H + Hk:])  # v untouched
    alone, none = f(cfg, x[:, :, :H].cuda(), None, pos[0].cuda())
    assert none is None and torch.equal(alone[0], qo[0])


def test_positions_at_the_ends_of_int32():
    """The turn is reduced in 64-bit integers: p = 2^31 - 1 is as good as 1
    up to the 2^-53 of the frequency (2^31 2^-53 turns, 1.5e-6 radians)."""
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_rotary_config(64)
    x = _inputs(1, 4, 2, 1, 64, torch.float32, 5)
    pos = torch.tensor([[[2 ** 31 - 1], [-2 ** 31], [0], [-1]]],
                       dtype=torch.int32)
    qo, _ = FV.rotary(cfg, x[:, :, :2].cuda(), None, pos.cuda())
    theta, mag = OR.frequencies([32])
    ref = OR.rotate(x[:, :, :2].double().numpy(), pos.numpy(), [32], theta,
                    mag, "interleaved")
    bound = 5e-6 * _partner(x[:, :, :2].double().numpy(), 32, "interleaved")
    assert (np.abs(qo.cpu().double().numpy() - ref) <= bound).all()


def test_gradient_matches_differences():
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_rotary_config(64, rotary_dim=48, layout="half",
                                scaling="yarn", factors=[4.0],
                                original_contexts=[64])
    x = _inputs(1, 6, 2, 1, 64, torch.float32, 6)[:, :, :2].contiguous()
    w = _inputs(1, 6, 2, 1, 64, torch.float32, 7)[:, :, :2].contiguous()
    pos = torch.arange(6, dtype=torch.int32).reshape(6, 1).cuda() * 50
    grad, _ = FV.rotary_bwd(cfg, w.cuda(), None, pos)
    f = lambda t: float((FV.rotary(cfg, t.cuda(), None, pos)[0].double().cpu()
                         * w.double()).sum())
    for idx in ((0, 0, 0, 0), (0, 3, 1, 30), (0, 5, 0, 47), (0, 5, 1, 63)):
        e = torch.zeros_like(x)
        e[idx] = 1.0  # the operator is linear: any step is exact
        diff = (f(x + e) - f(x - e)) / 2
        # 768 outputs, each within 1e-6 of its size
        assert abs(diff - float(grad[idx])) <= 768 * 1e-6


def test_strides_of_single_entries_and_broadcast_inputs():
    """A dimension of one entry may have any stride, and an input may repeat
    one token (stride 0)."""
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_rotary_config(64)
    x = _inputs(1, 1, 2, 1, 64, torch.bfloat16, 9).cuda()
    q = x[:, :, :2]
    odd = torch.as_strided(q, q.shape, (13, 7, 64, 1))  # one batch, one token
    pos = torch.tensor([[5]], dtype=torch.int32, device="cuda")
    assert torch.equal(FV.rotary(cfg, odd, None, pos)[0],
                       FV.rotary(cfg, q.contiguous(), None, pos)[0])
    wide = q.expand(3, 4, 2, 64)
    pos = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4, 1)
    assert torch.equal(FV.rotary(cfg, wide, None, pos)[0],
                       FV.rotary(cfg, wide.contiguous(), None, pos)[0])
    with pytest.raises(FV.FastVRError):
        FV.rotary(cfg, wide, None, pos, out=(wide, None))


def test_other_stream_and_bad_tensors():
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_rotary_config(64)
    x = _inputs(1, 40, 4, 4, 64, torch.bfloat16, 8).cuda()
    q, k = x[:, :, :4], x[:, :, 4:8]
    pos = torch.arange(40, dtype=torch.int32, device="cuda").reshape(40, 1)
    ref = FV.rotary(cfg, q, k, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = FV.rotary(cfg, q, k, pos)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    for bad in (dict(q=q.half()), dict(q=q[..., :32]), dict(q=q.cpu()),
                dict(k=k[:, :20]), dict(k=k.float()), dict(p=pos.long()),
                dict(p=pos[:20]), dict(p=pos.cpu()), dict(p=pos.reshape(-1)),
                dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)),
                dict(out=(q[:, :20], k)), dict(out=(q, None))):
        a = {**dict(q=q, k=k, p=pos, out=None), **bad}
        with pytest.raises(ValueError):
            FV.rotary(cfg, a["q"], a["k"], a["p"], out=a["out"])
