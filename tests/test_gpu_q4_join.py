"""Attention of few rows over a long 4-bit cache: key ranges split over many
CTAs and joined, with every number of query rows that a row block can hold.

Reference: float64 softmax attention over the values that the cache returns.
Bound per element: the probabilities are rounded to bfloat16, 2^-9 of each
term, and the output once more, 2^-9 of it; the float32 sums add less than a
tenth of that.  2^-8 of sum p |v| and of |o| leaves a factor of two.  The
log-sum-exp is a float32 sum of unrounded terms, its scores lose less than
2^-20 of |q||k| scale < 40: 1e-4."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 7, 8, 9, 16, 17, 25, 32])
@pytest.mark.parametrize("batch,heads,keys,d", [(1, 1, 20000, 128),
                                                (3, 2, 5000, 64),
                                                (2, 12, 3001, 128)])
def test_rows_and_parts(rows, batch, heads, keys, d):
    from paper_2609_36757_gb300 import fastvr as FV
    chunks = keys // rows
    T = chunks * rows
    g = torch.Generator("cuda").manual_seed(rows)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    k, v = rnd(batch, T, heads, d), rnd(batch, T, heads, d)
    q = 3 * rnd(batch, rows, heads, d)
    att = FV.StreamingAttention4(
        FV.make_config(batch, heads, d, rows, 1, chunks - 1))
    att.append(k, v)
    whole = FV.StreamingAttention4(FV.make_config(batch, heads, d, T, 1, 0))
    whole.append(k, v)
    kk, vv = (t.double().transpose(1, 2) for t in whole.read())
    before = att.launch_count()
    o, lse = att.forward(q, want_lse=True)
    assert att.launch_count() == before + 1  # straight over the codes
    s = q.double().transpose(1, 2) @ kk.transpose(2, 3) / d ** 0.5
    p = s.softmax(-1)
    want = (p @ vv).transpose(1, 2)
    size = (p @ vv.abs()).transpose(1, 2)
    err = (o.double() - want).abs()
    assert (err <= 2.0 ** -8 * (size + want.abs())).all()
    assert ((lse.double() - s.logsumexp(-1)).abs() <= 1e-4).all()
    assert torch.equal(att.forward(q), o)  # whichever CTA joins
