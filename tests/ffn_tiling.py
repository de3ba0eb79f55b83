"""The gated feed-forward's division of tiles (csrc/ffn_tiles.h), compiled for the
host and called through ctypes."""
import ctypes
import functools
import os
import subprocess
import tempfile
from typing import NamedTuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36757_gb300", "csrc")
SMS = 152

CODE = r"""
#include "ffn_tiles.h"
using namespace fastvr::ffn;
// Tiles of all pairs in turn, 8 ints each: pair, kind, which, m0, n0, steps,
// narrow, 0; the number of them, and in shape the lists' mt, nt, narrow, kind.
extern "C" int tiles(int64_t tokens, int64_t dim, int64_t hidden, int what,
                     int sms, int most, int* out, int* shape) {
  int pairs = 0, n = 0;
  const Division d = what == 0
                         ? divide_fwd(tokens, dim, hidden, sms, &pairs)
                         : divide_bwd(tokens, dim, hidden, what == 1, sms, &pairs);
  for (int l = 0; l < 2; ++l) {
    const int s[4] = {d.tile[l].mt, d.tile[l].nt, d.tile[l].narrow, d.kind[l]};
    for (int i = 0; i < 4; ++i) *shape++ = s[i];
  }
  *shape++ = pairs;
  *shape++ = d.extra;
  for (int p = 0; p < pairs; ++p) {
    Work w;
    for (int i = 0; nth_tile(d, p, pairs, i, &w); ++i, ++n) {
      if (n >= most) return -1;
      const int t[8] = {p, w.kind, w.which, w.m0, w.n0, w.steps, w.narrow, 0};
      for (int e = 0; e < 8; ++e) *out++ = t[e];
    }
  }
  return n;
}
"""
FWD, DX, DW = 0, 1, 2

# Sizes (tokens, dim, hidden, activation) whose tiles are several to a pair, ragged at
# both edges, and what they reach at 152 SMs: narrow tiles of the forward, of dx and of
# dW; most tiles of a pair, forward and backward; the kind with the longer sums.
SIZES = [
    ((3180, 776, 2056, "silu"), (0, 0, 0), (3, 2), DX),
    ((3559, 1856, 320, "gelu_tanh"), (1, 0, 0), (1, 3), DW),
    ((525, 1704, 1856, "silu"), (0, 0, 0), (1, 3), DX),
    ((364, 1832, 1512, "gelu"), (1, 1, 0), (1, 3), DX),
    ((3689, 1744, 72, "silu"), (1, 0, 1), (1, 3), DW),
    ((1061, 1000, 2728, "gelu_tanh"), (0, 1, 0), (2, 3), DX),
    ((2300, 264, 4360, "silu"), (0, 1, 0), (5, 2), DX),
    ((40000, 72, 64, "silu"), (1, 0, 1), (3, 3), DW),
]


class Tile(NamedTuple):
    pair: int
    kind: int
    which: int
    m0: int
    n0: int
    steps: int
    narrow: int


class Tiling(NamedTuple):
    tiles: list      # of all pairs in turn
    narrow: dict     # kind: 0 or 1
    rows: dict       # kind: rows of tiles
    pairs: int
    extra: int       # rounds of the second list before its common ones

    def rounds(self):
        """Most tiles of a pair."""
        count = [0] * self.pairs
        for t in self.tiles:
            count[t.pair] += 1
        return max(count)


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "tiles.cpp"), os.path.join(d, "tiles.so")
        with open(src, "w") as f:
            f.write(CODE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I",
                        CSRC, src, "-o", lib], check=True)
        f = ctypes.CDLL(lib).tiles
    f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 3 + [
        ctypes.POINTER(ctypes.c_int)] * 2
    return f


@functools.lru_cache(maxsize=None)
def _room():
    return (ctypes.c_int * (8 << 17))()


def tiling(tokens, dim, hidden, what, sms=SMS):
    """what: "fwd", "bwd" or "frozen" (dx alone)."""
    out, shape = _room(), (ctypes.c_int * 10)()
    n = _lib()(tokens, dim, hidden, ("fwd", "bwd", "frozen").index(what), sms,
               len(out) // 8, out, shape)
    assert n >= 0
    tiles = [Tile(*out[8 * i:8 * i + 7]) for i in range(n)]
    lists = [shape[4 * i:4 * i + 4] for i in range(2)]
    if what == "fwd":
        lists = lists[:1]
    return Tiling(tiles, {k: s for _, _, s, k in lists},
                  {k: m for m, _, _, k in lists}, shape[8], shape[9])
