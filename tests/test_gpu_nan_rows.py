"""NaN in queries and keys where key ranges are split over CTAs and merged.

A row whose scores are all NaN, or some of them, is NaN in the output and in
the log-sum-exp, whichever parts the NaN lie in: it is not a row that sees no
key (zeros and -infinity).  Rows beside it keep their results: a score has
2^-20 of |q||k| scale < 20 and the output its usual roundings of the
probabilities and of itself, 2^-9 of sum p |v| < 6 each, doubled as the
running references may differ: 2e-5 and 2^-8 (6 + 6)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

NAN = float("nan")
N, CHUNKS, D = 200, 100, 64


def _run(four, q, k, v, first=None):
    """(o, lse) of the last chunk's queries; the launch is a split one."""
    from paper_2609_36757_gb300 import fastvr as FV
    B, _, H, _ = k.shape
    cfg = FV.make_config(B, H, D, N, 1, -1, CHUNKS)
    att = FV.StreamingAttention4(cfg) if four else FV.StreamingAttention(cfg)
    for c in range(CHUNKS):
        at = slice(c * N, (c + 1) * N)
        att.append(k[:, at].contiguous(), v[:, at].contiguous())
    before = att.launch_count()
    kw = {} if first is None else dict(first_chunk=first)
    out = att.forward(q, want_lse=True, **kw)
    # (read-back,) attention over parts of the keys, merge
    assert att.launch_count() == before + (3 if four else 2)
    assert att.status() == FV.FASTVR_OK
    return out


def _inputs(batch, heads, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda n: torch.randn(batch, n, heads, D, generator=g,
                                device="cuda").to(torch.bfloat16)
    return rnd(N), rnd(N * CHUNKS), rnd(N * CHUNKS)


def _same(a, b):
    (o, lse), (ro, rl) = a, b
    assert torch.isfinite(ro).all() and torch.isfinite(rl).all()
    assert ((o.float() - ro.float()).abs() <= 2.0 ** -8 * 12).all()
    assert ((lse - rl).abs() <= 2e-5).all()


@pytest.mark.parametrize("four,late", [(False, False), (True, False),
                                       (True, True)])
def test_nan_queries(four, late):
    q, k, v = _inputs(2, 2, 1)
    first = torch.tensor([3, CHUNKS], dtype=torch.int32,
                         device="cuda") if late else None
    ref = _run(four, q, k, v, first)
    bad = q.clone()
    rows = [5, 77, N - 1]
    bad[:, rows, 1, 9] = NAN
    o, lse = _run(four, bad, k, v, first)
    sees = [0] if late else [0, 1]
    for b in sees:
        assert torch.isnan(o[b, rows, 1]).all()
        assert torch.isnan(lse[b, 1, rows]).all()
    if late:  # entry 1 has not joined: its rows see no key, NaN or not
        assert (o[1] == 0).all() and (lse[1] == -torch.inf).all()
    rest = [r for r in range(N) if r not in rows]
    for h, keep in ((0, list(range(N))), (1, rest)):
        _same((o[sees][:, keep, h], lse[sees][:, h, keep]),
              (ref[0][sees][:, keep, h], ref[1][sees][:, h, keep]))


@pytest.mark.parametrize("four,late", [(False, False), (True, False),
                                       (True, True)])
# all keys; the first 64 tiles of 128, which is sixteen whole parts of 157 // 4
# (what the merge takes at once); half of them; one
@pytest.mark.parametrize("at", [slice(0, None), slice(0, 64 * 128),
                                slice(0, N * CHUNKS // 2),
                                slice(N * CHUNKS // 2, None),
                                slice(12345, 12346)])
def test_nan_keys(four, late, at):
    q, k, v = _inputs(1, 1, 2)
    first = torch.tensor([-1], dtype=torch.int32,
                         device="cuda") if late else None
    k[:, at] = NAN
    o, lse = _run(four, q, k, v, first)
    assert torch.isnan(o).all() and torch.isnan(lse).all()
