"""The 4-bit cache and its attention on the GPU against the float64 oracle.

The quantiser is exact by definition: read-back values equal the oracle's bit
for bit.  Attention: P enters the tensor cores in bfloat16 (2^-9 of each term)
and the output is rounded once more (2^-9), so an element is within 2^-9
(sum p |v| + |o|); the scores (fp32 sums of exact products, d <= 128 terms)
and exponentials add less than 1e-5 (1 + max |score|) of sum p |v|.  With a
factor of two on the roundings:  2^-8 (sum p |v| + |o|) + 2e-5 (1 + max |s|)
sum p |v|.  The log-sum-exp: 2e-5 (1 + max |s|)."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import q4 as Q4

pytestmark = pytest.mark.gpu


def f64(t):
    return t.cpu().double().numpy()


@dataclasses.dataclass
class Case:
    B: int
    H: int
    Hk: int
    d: int
    N: int
    k: int
    W: int
    chunks: int
    last: int = 0        # frames of the last chunk (0: k)
    max_chunks: int = 0
    rows: int = 0        # query rows checked per (b, h); 0: all

    def cfg(self, FV):
        return FV.make_config(self.B, self.H, self.d, self.N, self.k, self.W,
                              self.max_chunks or (self.chunks
                                                  if self.W < 0 else 0))

    def frames(self, c):
        return self.last if self.last and c == self.chunks - 1 else self.k


def stream(case, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    for c in range(case.chunks):
        L = case.frames(c) * case.N
        q, = (torch.randn(case.B, L, case.H, case.d, generator=g) * scale,)
        k, v = torch.randn(2, case.B, L, case.Hk, case.d, generator=g)
        k[..., :3] *= 6.0  # strong channels
        yield c, *(t.to(torch.bfloat16) for t in (q, k, v))


def check_attention(case, c, q, o, lse, kv, first=None, scale=None, seed=0):
    """kv: the cache values of the visible window, oldest first: two lists of
    [B, L, Hk, d]."""
    kk, vv = (np.concatenate(t, 1) for t in kv)
    lo = 0 if case.W < 0 else max(0, c - case.W)
    chunk = np.concatenate([np.full(t.shape[1], lo + i)
                            for i, t in enumerate(kv[0])])
    q, o, lse = f64(q), f64(o), f64(lse)
    rows = np.arange(q.shape[1])
    if case.rows and case.rows < len(rows):
        rows = np.unique(np.concatenate([
            [0, len(rows) - 1],
            np.random.default_rng(seed).integers(0, len(rows), case.rows)]))
    for b in range(case.B):
        vis = chunk >= (lo if first is None else first[b])
        ref, rl, mass, top = Q4.attention(
            q[b][rows], kk[b], vv[b], scale or case.d ** -0.5, vis)
        if not vis.any():
            assert (o[b] == 0).all() and (lse[b] == -np.inf).all()
            continue
        t = (1 + top.T)[..., None]  # [rows, H, 1]
        bound = 2.0 ** -8 * (mass + np.abs(ref)) + 2e-5 * t * mass
        err = np.abs(o[b][rows] - ref)
        assert (err <= bound).all(), (b, float((err / bound).max()))
        lerr = np.abs(lse[b][:, rows] - rl)
        assert (lerr <= 2e-5 * (1 + top)).all(), float(lerr.max())


CASES = [
    Case(1, 1, 1, 128, 1, 1, -1, 3),                 # single tokens
    Case(2, 4, 2, 64, 1, 1, 5, 40),                  # ring wraps many times
    Case(1, 12, 12, 128, 1, 1, 299, 330),
    Case(3, 8, 1, 128, 1, 1, 40, 97),                # 8 heads share one
    Case(1, 32, 2, 64, 1, 1, 64, 130),               # 16 share one
    Case(1, 24, 1, 128, 1, 1, 33, 60),               # 24 rows: ragged block
    Case(1, 2, 2, 128, 3, 3, 2, 9, last=1),          # 9 rows, ragged last
    Case(2, 3, 3, 64, 17, 1, 3, 7),                  # 17 rows
    Case(1, 2, 1, 128, 37, 2, 1, 4),                 # 148 rows
    Case(1, 2, 2, 128, 300, 2, -1, 4, rows=90),
    Case(1, 2, 2, 64, 111, 3, 4, 9, last=2, rows=90),
    Case(2, 4, 2, 128, 257, 2, 1, 4, rows=60),       # shared heads, long
    Case(1, 12, 12, 128, 1590, 2, 2, 4, rows=20),    # 480p frames
    Case(1, 4, 4, 128, 5, 1, 0, 3),                  # no window
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_stream(i):
    """Chunk by chunk: what is stored, and the attention over it."""
    from paper_2609_36757_gb300 import fastvr as FV
    case = CASES[i]
    att = FV.StreamingAttention4(case.cfg(FV), kv_heads=case.Hk)
    # stale contents must never matter: scales of NaN, codes of anything
    att.cache.fill_(0xff)
    att.workspace.fill_(0xff)
    window = []
    for c, q, k, v in stream(case, 500 + i):
        att.append(k.cuda(), v.cuda())
        kr, vr = att.read()
        want = [Q4.values(f64(t)) for t in (k, v)]
        assert np.array_equal(f64(kr), want[0])
        assert np.array_equal(f64(vr), want[1])
        window.append(want)
        if case.W >= 0:
            window = window[-(case.W + 1):]
        few = case.chunks > 20 and c % 13 and c < case.chunks - 2
        o, lse = att.forward(q.cuda(), want_lse=True)
        if not few:
            check_attention(case, c, q, o, lse, list(zip(*window)), seed=c)
            o2 = att.forward(q.cuda())  # repeated, without lse: bit for bit
            assert torch.equal(o2, o)
    assert att.status() == FV.FASTVR_OK


@pytest.mark.parametrize("keys", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65,
                                  127, 255, 257, 1000])
@pytest.mark.parametrize("d", [64, 128])
def test_every_tile_edge(keys, d):
    """One query token over `keys` tokens, whatever lies behind them."""
    from paper_2609_36757_gb300 import fastvr as FV
    case = Case(1, 3, 3, d, 1, 1, 1030, keys)
    att = FV.StreamingAttention4(case.cfg(FV), kv_heads=3)
    att.cache.fill_(0xff)
    g = torch.Generator().manual_seed(keys)
    k, v = torch.randn(2, 1, keys, 3, d, generator=g).to(torch.bfloat16)
    q = torch.randn(1, 1, 3, d, generator=g).to(torch.bfloat16)
    # start late in the ring, so that the keys wrap
    att.set_state(1031 * 3 - keys // 2, 1)
    att.append(k.cuda(), v.cuda())  # `keys` whole chunks at once
    c = att.state()[0] - 1
    first = c - keys + 1  # what lies before was never written
    o, lse = att.forward(q.cuda(), want_lse=True, first_chunk=torch.tensor(
        [first], dtype=torch.int32, device="cuda"))
    vals = [Q4.values(f64(t)) for t in (k, v)]
    ref, rl, mass, top = Q4.attention(f64(q)[0], vals[0][0], vals[1][0],
                                      d ** -0.5, np.ones(keys, bool))
    bound = 2.0 ** -8 * (mass + np.abs(ref)) + 2e-5 * (
        1 + top.T[..., None]) * mass
    assert (np.abs(f64(o)[0] - ref) <= bound).all()
    assert (np.abs(f64(lse)[0] - rl) <= 2e-5 * (1 + top)).all()


@pytest.mark.parametrize("N,k", [(1, 1), (7, 2), (150, 2)])
def test_streams_that_joined_late(N, k):
    """first_chunk hides a batch entry's earlier chunks, NaN and infinities
    among them; an entry that has not joined yet gets zeros and -inf."""
    from paper_2609_36757_gb300 import fastvr as FV
    case = Case(6, 4, 2, 128, N, k, 4, 9, rows=40)
    att = FV.StreamingAttention4(case.cfg(FV), kv_heads=2)
    att.cache.fill_(0xff)
    first = [-5, 0, 6, 8, 9, 2 ** 31 - 1]  # c = 8: the last two see nothing
    window = []
    for c, q, kk, vv in stream(case, 77):
        for b, f in enumerate(first):
            if c < f:
                kk[b, ::2], vv[b, 1::2] = float("nan"), float("inf")
                vv[b, ::3], kk[b, 1::3] = -float("inf"), 3e38
        att.append(kk.cuda(), vv.cuda())
        window = (window + [[Q4.values(f64(t)) for t in (kk, vv)]])[-5:]
    dev = torch.tensor(first, dtype=torch.int32, device="cuda")
    o, lse = att.forward(q.cuda(), first_chunk=dev, want_lse=True)
    check_attention(case, 8, q, o, lse, list(zip(*window)), first=first)
    # without the mask the NaN of entry 2 onwards do reach the result
    o = att.forward(q.cuda())
    assert torch.isfinite(o[:2].float()).all()
    assert torch.isnan(o[2].float()).any()


def test_quantiser_over_all_mantissas():
    """Every mantissa of a group's maximum with every value mantissa down to
    2^-5 of it, both signs, through the append and the read-back."""
    from paper_2609_36757_gb300 import fastvr as FV
    vals = np.concatenate([np.arange(128, 256) / 128.0 * 2.0 ** -e
                           for e in range(6)])
    groups = []
    for top in np.arange(128, 256) / 128.0:
        ok = vals[vals <= top]
        ok = np.concatenate([ok, -ok])
        ok = np.concatenate([ok, np.zeros(-len(ok) % 31)]).reshape(-1, 31)
        groups.append(np.concatenate([np.full((len(ok), 1), top), ok], 1))
    x = np.concatenate(groups)
    for shift in (0, -90, 100):  # the exponent does not matter
        y = (x * 2.0 ** shift).reshape(-1)
        y = np.concatenate([y, np.zeros(-len(y) % (2 * 128))])
        t = torch.from_numpy(y).to(torch.bfloat16).reshape(1, -1, 2, 128)
        assert np.array_equal(f64(t).reshape(-1), y)
        cfg = FV.make_config(1, 2, 128, t.shape[1], 1, 0)
        att = FV.StreamingAttention4(cfg)
        att.append(t.cuda(), (-t).cuda())
        k, v = att.read()
        want = Q4.values(f64(t))
        assert np.array_equal(f64(k), want)
        assert np.array_equal(f64(v), -want)


def test_quantiser_ends_of_the_range():
    from paper_2609_36757_gb300 import fastvr as FV
    x = torch.zeros(1, 8, 1, 64)
    nan, inf = float("nan"), float("inf")
    for t, v in enumerate((2.0 ** -100, 2.0 ** -101, 2.0 ** 119, 2.0 ** 120,
                           inf, -inf, nan, 1e-40)):
        x[0, t, 0, 5] = v
        x[0, t, 0, 7] = 2.0 ** -102
        x[0, t, 0, 40] = 1.0
    x = x.to(torch.bfloat16)
    att = FV.StreamingAttention4(FV.make_config(1, 1, 64, 8, 1, 0))
    att.append(x.cuda(), x.cuda())
    k, v = att.read()
    want = Q4.values(f64(x))
    assert np.array_equal(f64(k), want, equal_nan=True)
    assert np.array_equal(f64(v), want, equal_nan=True)
    assert np.isnan(want[0, 3:7, 0, :32]).all() and want[0, 6, 0, 40] != 0


def test_strides_prefix_state_and_streams():
    """Slices of a fused projection, several chunks at once, a resumed plan
    on the same cache, another stream: bit for bit the same."""
    from paper_2609_36757_gb300 import fastvr as FV
    case = Case(2, 4, 2, 64, 19, 2, 3, 6)
    cfg = case.cfg(FV)
    chunks = list(stream(case, 9))
    ref = FV.StreamingAttention4(cfg, kv_heads=2)
    for _, q, k, v in chunks:
        ref.append(k.cuda(), v.cuda())
    o = ref.forward(q.cuda())

    big = torch.cat([torch.cat([k, v], 2) for _, _, k, v in chunks[2:]], 1)
    big = big.cuda()  # [B, 4 chunks, 2 Hk, d]
    att = FV.StreamingAttention4(cfg, kv_heads=2, workspace=ref.workspace)
    att.set_state(2, 2)
    att.append(big[:, :, :2], big[:, :, 2:])
    assert att.state() == (6, 2)
    assert torch.equal(att.forward(q.cuda()), o)
    for c in (2, 3, 4, 5):
        for a, b in zip(att.read(c), ref.read(c)):
            assert torch.equal(a, b)

    resumed = FV.StreamingAttention4(cfg, kv_heads=2)
    resumed.cache.copy_(ref.cache)
    resumed.set_state(*ref.state())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    qd = q.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = resumed.forward(qd)
    side.synchronize()
    # the first device call clears the control block on its own stream
    assert torch.equal(got, o)
    with pytest.raises(FV.FastVRError):
        att.read(1)
    with pytest.raises(ValueError):
        att.forward(q[:, :19].cuda())
    with pytest.raises(ValueError):
        att.forward(qd, first_chunk=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError):
        att.append(big[:, :38, :2], big[:, :38, :1])
    with pytest.raises(ValueError):
        att.append(big[:, :38, :2].half(), big[:, :38, 2:])


def test_offsets_past_32_bits():
    """A cache whose last head starts 4.3 GB into the codes: the newest
    tokens of every head are stored and read at the right place."""
    from paper_2609_36757_gb300 import fastvr as FV
    Hk, d, T = 8, 128, 9_000_001
    cfg = FV.make_config(1, Hk, d, 1, 1, -1, T)
    att = FV.StreamingAttention4(cfg)
    n = 300
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(2, 1, n, Hk, d, generator=g).to(torch.bfloat16)
    q = torch.randn(1, 1, Hk, d, generator=g).to(torch.bfloat16)
    att.set_state(T - n, 1)
    att.append(k.cuda(), v.cuda())
    first = torch.tensor([T - n], dtype=torch.int32, device="cuda")
    o, lse = att.forward(q.cuda(), first_chunk=first, want_lse=True)
    vals = [Q4.values(f64(t)) for t in (k, v)]
    ref, rl, mass, top = Q4.attention(f64(q)[0], vals[0][0], vals[1][0],
                                      d ** -0.5, np.ones(n, bool))
    bound = 2.0 ** -8 * (mass + np.abs(ref)) + 2e-5 * (
        1 + top.T[..., None]) * mass
    assert (np.abs(f64(o)[0] - ref) <= bound).all()
    kr, vr = att.read(T - 7)
    assert np.array_equal(f64(kr)[0, 0], vals[0][0, n - 7])
    assert np.array_equal(f64(vr)[0, 0], vals[1][0, n - 7])
    assert att.status() == FV.FASTVR_OK


def test_workspace_offsets_past_32_bits():
    """A chunk of 350 queries over 700 000 tokens of 24 heads: the expanded
    keys take 2.15e9 elements.  The newest chunks, checked on the last head."""
    from paper_2609_36757_gb300 import fastvr as FV
    H, d, N, chunks, seen = 24, 128, 350, 2000, 3
    cfg = FV.make_config(1, H, d, N, 1, -1, chunks)
    att = FV.StreamingAttention4(cfg)
    assert H * d * N * chunks > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(6)
    tail = torch.randn(2, 1, seen * N, H, d, generator=g,
                       device="cuda").to(torch.bfloat16)
    att.cache.zero_()
    att.set_state(chunks - seen, 1)
    att.append(tail[0], tail[1])
    q = torch.randn(1, N, H, d, generator=g, device="cuda").to(torch.bfloat16)
    for first, lo in ((chunks - seen, 0), (chunks - 1, 2 * N)):
        o, lse = att.forward(q, want_lse=True, first_chunk=torch.tensor(
            [first], dtype=torch.int32, device="cuda"))
        kk, vv = (Q4.values(f64(t[0, lo:, -1:])) for t in tail)
        ref, rl, mass, top = Q4.attention(f64(q[0, ::50, -1:]), kk, vv,
                                          d ** -0.5, np.ones(len(kk), bool))
        bound = 2.0 ** -8 * (mass + np.abs(ref)) + 2e-5 * (
            1 + top.T[..., None]) * mass
        assert (np.abs(f64(o[0, ::50, -1:]) - ref) <= bound).all()
        assert (np.abs(f64(lse[0, -1:, ::50]) - rl) <= 2e-5 * (1 + top)).all()
    # everything visible: the zeros before count 1 each in the sum
    o, lse = att.forward(q, want_lse=True)
    s = f64(q[0, ::50, -1]) @ Q4.values(f64(tail[0][0, :, -1])).T * d ** -0.5
    want = np.log((chunks - seen) * N + np.exp(s).sum(-1))
    assert np.abs(f64(lse[0, -1, ::50]) - want).max() <= 2e-5 * (
        1 + np.abs(s).max())
    assert att.status() == FV.FASTVR_OK


def test_output_is_not_the_query():
    from paper_2609_36757_gb300 import fastvr as FV
    att = FV.StreamingAttention4(FV.make_config(1, 2, 64, 1, 1, 3))
    t = torch.ones(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    att.append(t, t)
    with pytest.raises(ValueError):
        att.forward(t, out=t)


def test_peaked_and_flat_rows():
    """Large scores (the reference moves often) and Q = 0 (the mean of V)."""
    from paper_2609_36757_gb300 import fastvr as FV
    case = Case(1, 2, 2, 128, 1, 1, -1, 700)
    att = FV.StreamingAttention4(case.cfg(FV))
    g = torch.Generator().manual_seed(4)
    k, v = torch.randn(2, 1, 700, 2, 128, generator=g).to(torch.bfloat16)
    att.append((k.float() * torch.linspace(0.1, 9, 700)[None, :, None, None])
               .to(torch.bfloat16).cuda(), v.cuda())
    vals_v = Q4.values(f64(v))
    zero = torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16, device="cuda")
    o, lse = att.forward(zero, want_lse=True)
    assert np.allclose(f64(lse), np.log(700), atol=2e-5)
    assert np.abs(f64(o)[0, 0] - vals_v[0].mean(0)).max() <= 2.0 ** -8
    vals_k = Q4.values(f64((k.float() * torch.linspace(0.1, 9, 700)[
        None, :, None, None]).to(torch.bfloat16)))
    q = (8 * torch.randn(1, 1, 2, 128, generator=g)).to(torch.bfloat16)
    o, lse = att.forward(q.cuda(), want_lse=True)
    check_attention(case, 699, q, o, lse, ([vals_k], [vals_v]))


def test_debug_library_checks_pass():
    """The index checks of the debug build report nothing, and its results
    are the release build's."""
    from paper_2609_36757_gb300 import fastvr as FV
    case = Case(2, 4, 2, 128, 70, 2, 2, 5, last=1)

    def run():
        att = FV.StreamingAttention4(case.cfg(FV), kv_heads=2)
        outs = []
        for _, q, k, v in stream(case, 11):
            att.append(k.cuda(), v.cuda())
            outs += [att.forward(q.cuda()), *att.read()]
        assert att.status() == FV.FASTVR_OK
        return outs

    ref = run()
    previous = FV.use_library(FV.DEBUG_LIB_PATH)
    try:
        got = run()
    finally:
        FV.lib = previous
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
