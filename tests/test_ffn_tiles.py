"""The feed-forward's tiles: the pairs' shares hold every tile once, and cover the
results exactly."""
import random

import pytest

from ffn_tiling import DW, DX, FWD, SIZES, tiling


def _check(tokens, dim, hidden, sms):
    want_steps = {FWD: -(-dim // 64), DX: 2 * -(-hidden // 64),
                  DW: -(-tokens // 64)}
    size = {FWD: (tokens, hidden), DX: (tokens, dim), DW: (hidden, dim)}
    for what, kinds in (("fwd", [(FWD, 0)]), ("frozen", [(DX, 0)]),
                        ("bwd", [(DX, 0), (DW, 0), (DW, 1)])):
        t = tiling(tokens, dim, hidden, what, sms)
        assert 1 <= t.pairs <= max(1, sms // 2)
        for kind, which in kinds:
            rows, cols = size[kind]
            across = (128 if kind == FWD else 256) >> t.narrow[kind]
            want = [(m, n) for m in range(0, rows, 256)
                    for n in range(0, cols, across)]
            got = [(x.m0, x.n0) for x in t.tiles
                   if (x.kind, x.which) == (kind, which)]
            assert sorted(got) == want, (what, kind, which)
        assert {(x.kind, x.which) for x in t.tiles} == set(kinds)
        assert all(x.steps == want_steps[x.kind] and
                   x.narrow == t.narrow[x.kind] for x in t.tiles)
        # no pair is left without work
        assert {x.pair for x in t.tiles} == set(range(t.pairs))


@pytest.mark.parametrize("sms", [2, 7, 148, 152])
def test_every_tile_once(sms):
    rng = random.Random(sms)
    log = lambda lo, hi: round(lo * (hi / lo) ** rng.random())
    for _ in range(150):
        _check(log(1, 20000), 8 * log(1, 300), 8 * log(1, 900), sms)


@pytest.mark.parametrize("sizes", [(1, 8, 8), (33, 8, 8), (256, 256, 256),
                                   (257, 264, 264), (16320, 1536, 4096),
                                   (2049, 520, 1032), (3180, 776, 2056),
                                   (1061, 1000, 2728), (100000, 64, 64),
                                   (40, 2048, 5632)])
def test_every_tile_once_at(sizes):
    _check(*sizes, 152)


@pytest.mark.parametrize("case", SIZES, ids=lambda c: str(c[0]))
def test_sizes_of_the_gpu_tests_reach_what_they_are_for(case):
    (tokens, dim, hidden, _), narrow, rounds, first = case
    f, b = (tiling(tokens, dim, hidden, what) for what in ("fwd", "bwd"))
    assert (f.narrow[FWD], b.narrow[DX], b.narrow[DW]) == narrow
    assert (f.rounds(), b.rounds()) == rounds
    assert b.tiles[0].kind == first


def test_sizes_of_the_gpu_tests_cover_the_kernel():
    """Each kind wide and narrow with its tiles following one another in both halves of
    TMEM and again in the first, more row tiles than share their columns, and the
    longer sums' pairs making up for others."""
    reach = [(f, b) for f, b in ((tiling(*c[0][:3], "fwd"),
                                  tiling(*c[0][:3], "bwd")) for c in SIZES)]
    assert any(not f.narrow[FWD] and f.rounds() >= 3 and f.rows[FWD] > 8
               for f, _ in reach)
    assert any(f.narrow[FWD] and f.rounds() >= 2 for f, _ in reach)
    for dx, dw in ((0, 0), (1, 0), (0, 1)):
        assert any((b.narrow[DX], b.narrow[DW]) == (dx, dw) and
                   b.rounds() >= 3 for _, b in reach)
    assert any(not b.narrow[DX] and b.rows[DX] > 8 for _, b in reach)
    assert any(not b.narrow[DW] and b.rows[DW] > 8 for _, b in reach)
    assert any(b.extra >= 2 for _, b in reach)
