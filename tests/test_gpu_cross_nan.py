"""NaN and infinities that the attention sees: a NaN in a query, key or value is
NaN in every result that the formulas take it to, whatever the token's index, and
in no other; a row whose scores are all -infinity is 0 / 0."""
import pytest
import torch

pytestmark = pytest.mark.gpu

NAN = float("nan")
T, LEN = 300, 270  # keys, of which the last ones are not seen


def _inputs(L, d, seed=1):
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g,
                                 device="cuda").to(torch.bfloat16)
    return rnd(1, L, 4, d), rnd(1, T, 2, d), rnd(1, T, 2, d), rnd(1, L, 4, d)


def _run(q, k, v, do, kv_len):
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_cross_config()
    out, lse = FV.cross_attention(cfg, q, k, v, kv_len, want_lse=True)
    g = FV.cross_attention_bwd(cfg, q, k, v, out, do, lse, kv_len)
    return dict(out=out, lse=lse.transpose(1, 2), dq=g.dq, dk=g.dk, dv=g.dv)


def _len(cut):
    return torch.tensor([LEN], dtype=torch.int32,
                        device="cuda") if cut else None


def _expect(got, clean, nan):
    """got is NaN at `nan` (name: index or None) and clean's bits elsewhere."""
    for name, t in got.items():
        where = torch.zeros_like(t, dtype=torch.bool)
        if name in nan:
            where[nan[name]] = True
        assert bool(torch.isnan(t[where]).all()), name
        assert torch.equal(t[~where], clean[name][~where]), name


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,cut", [(1, True), (8, False), (300, False),
                                   (300, True)])
def test_nan_query_at_any_index(L, cut, d):
    q, k, v, do = _inputs(L, d)
    kv_len = _len(cut)
    clean = _run(q, k, v, do, kv_len)
    seen = slice(0, LEN if cut else T)
    # query head 2 is one of the two over key head 1
    for i in range(L if L < 128 else 32):
        row = i if L < 128 else 128 + i
        bad = q.clone()
        bad[0, row, 2, 5] = NAN
        at = (0, row, 2)
        _expect(_run(bad, k, v, do, kv_len), clean,
                dict(out=at, lse=at, dq=at, dk=(0, seen, 1), dv=(0, seen, 1)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L", [2, 300])
def test_nan_key_and_value(L, d):
    q, k, v, do = _inputs(L, d)
    kv_len = _len(True)
    clean = _run(q, k, v, do, kv_len)
    seen = slice(0, LEN)
    for t in (0, 31, 130, LEN - 1):
        bad = k.clone()
        bad[0, t, 1, 7] = NAN
        at = (0, slice(None), slice(2, 4))
        _expect(_run(q, bad, v, do, kv_len), clean,
                dict(out=at, lse=at, dq=at, dk=(0, seen, 1), dv=(0, seen, 1)))
        bad = v.clone()
        bad[0, t, 1, 7] = NAN
        # D = <dout, out> is NaN in every row, so dS is, but not P
        got = _run(q, k, bad, do, kv_len)
        _expect(got, clean, dict(out=at + (7,), dq=at, dk=(0, seen, 1)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,row", [(1, 0), (7, 3), (300, 1), (300, 29),
                                   (300, 299)])
def test_row_of_minus_infinities(L, row, d):
    q, k, v, do = _inputs(L, d)
    k[..., 9] = -k[..., 9].abs() - 0.5  # below zero
    kv_len = _len(True)
    clean = _run(q, k, v, do, kv_len)
    bad = q.clone()
    bad[0, row, 0, 9] = float("inf")
    got = _run(bad, k, v, do, kv_len)
    assert float(got["lse"][0, row, 0]) == -float("inf")
    got["lse"][0, row, 0] = clean["lse"][0, row, 0]
    seen = slice(0, LEN)
    _expect(got, clean, dict(out=(0, row, 0), dq=(0, row, 0),
                             dk=(0, seen, 0), dv=(0, seen, 0)))


@pytest.mark.parametrize("d", [64, 128])
def test_one_shot_backward_nan_query_at_any_index(d):
    """One chunk: every key sees the row."""
    from paper_2609_36757_gb300 import fastvr as FV
    n = 512
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v, do = (torch.randn(1, n, 2, d, generator=g, device="cuda").to(
        torch.bfloat16) for _ in range(4))
    cfg = FV.make_config(1, 2, d, n, 1)

    def run(q):
        out, lse = FV.blockcausal_attention(cfg, q, k, v, want_lse=True)
        r = FV.blockcausal_attention_bwd(cfg, q, k, v, out, do, lse)
        return dict(dq=r[0], dk=r[1], dv=r[2])

    clean = run(q)
    everything = (0, slice(None), 1)
    for i in range(32):
        bad = q.clone()
        bad[0, 256 + i, 1, 3] = NAN
        _expect(run(bad), clean, dict(dq=(0, 256 + i, 1), dk=everything,
                                      dv=everything))
