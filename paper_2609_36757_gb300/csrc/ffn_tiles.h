// How the gated feed-forward's tiles are divided among pairs of CTAs
// (gated_ffn.cu): host code, and the kernel's walk through its share.
#pragma once

#include <stdint.h>

#include <algorithm>

#ifdef __CUDACC__
#define FASTVR_HD __host__ __device__
#else
#define FASTVR_HD
#endif

namespace fastvr {
namespace ffn {

constexpr int kHalf = 128;      // rows of A and of B in one CTA
constexpr int kStep = 64;       // of the summed axis in one stage
constexpr int kGroupTiles = 8;  // row tiles that share their columns' tiles

enum Kind { kFwd, kDx, kDw };

// Tiles of one kind: results [rows, cols], rows of tiles by tiles across.
struct Tiles {
  int32_t rows, cols, mt, nt, count, steps;
  int32_t narrow;  // 128 columns of results instead of 256
};

// Two lists of tiles: the forward's are all in the first; the backward's are those
// with the longer sums, and the others.
struct Division {
  Tiles tile[2];
  int32_t kind[2];
  // Pairs from `heavy` on (0: all) have one tile fewer of the first list than the
  // others and take `extra` of the second list before its common rounds.
  int32_t heavy, extra;
};

FASTVR_HD inline int imin(int a, int b) { return a < b ? a : b; }

// The i-th tile of a pair of CTAs; false behind its last.
struct Work {
  int kind, m0, n0, steps, which, narrow;  // which: dWg or dWu
};
FASTVR_HD inline bool nth_tile(const Division& p, int pair, int pairs, int i,
                               Work* w) {
  int list = 0, t = pair + i * pairs;
  if (t >= p.tile[0].count) {
    list = 1;
    i -= (p.tile[0].count + pairs - 1 - pair) / pairs;  // had of the first
    const int light = pairs - p.heavy;
    const int ahead = imin(p.tile[1].count, p.extra * light);
    if (p.extra > 0 && pair >= p.heavy && i < p.extra) {
      t = pair - p.heavy + i * light;
      if (t >= ahead) return false;
    } else {
      if (p.extra > 0 && pair >= p.heavy) i -= p.extra;
      // common rounds, the pairs with fewer tiles of the first list first
      t = ahead + (pair >= p.heavy ? pair - p.heavy : pair + light) + i * pairs;
    }
    if (t >= p.tile[1].count) return false;
  }
  const Tiles& a = p.tile[list];
  w->kind = p.kind[list];
  w->steps = a.steps;
  w->narrow = a.narrow;
  w->which = 0;
  if (w->kind == kDw) {
    const int one = a.mt * a.nt;
    w->which = t >= one;
    t -= w->which * one;
  }
  const int across = kGroupTiles * a.nt;
  const int first = t / across * kGroupTiles;
  const int gm = imin(kGroupTiles, a.mt - first), r = t % across;
  w->m0 = (first + r % gm) * 2 * kHalf;
  w->n0 = r / gm * ((w->kind == kFwd ? kHalf : 2 * kHalf) >> w->narrow);
  return true;
}

inline int up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// `wide`: columns of a wide tile.
inline Tiles make_tiles(int64_t rows, int64_t cols, int wide, int copies, int steps,
                        int narrow) {
  Tiles t;
  t.rows = (int32_t)rows;
  t.cols = (int32_t)cols;
  t.mt = up(rows, 2 * kHalf);
  t.nt = up(cols, wide >> narrow);
  t.count = t.mt * t.nt * copies;
  t.steps = steps;
  t.narrow = narrow;
  return t;
}

// The pairs' shares of two lists of tiles, and the time of the pair that ends
// last in steps of wide tiles.  A narrow tile has half of the products but three
// quarters of the loads, which bound it.
struct Shares {
  int pairs, heavy, extra;
  double time;
};
inline Shares share(const Tiles& a, const Tiles& b, int sms) {
  const int pairs = std::min(sms / 2, a.count + b.count);
  const double ca = (a.steps + 8) * (a.narrow ? 0.75 : 1.0);
  const double cb = (b.steps + 8) * (b.narrow ? 0.75 : 1.0);
  const int heavy = a.count % pairs, light = pairs - heavy;
  Shares best = {pairs, heavy, 0, 0.0};
  // extra rounds that make up for a tile of the first list, or one more
  const int most = b.count > 0 && heavy > 0 ? (int)(ca / cb) + 1 : 0;
  for (int extra = std::max(0, most - 1); extra <= most; ++extra) {
    const int ahead = (int)std::min<int64_t>(b.count, (int64_t)extra * light);
    double time = 0.0;
    for (int p = 0; p < pairs; ++p) {
      const int own = p >= heavy ? p - heavy : p + light;
      int64_t n = (b.count - ahead + pairs - 1 - own) / pairs;
      if (extra > 0 && p >= heavy)
        n += std::min(extra, (ahead - own + light - 1) / light);
      time = std::max(time,
                      (a.count + pairs - 1 - p) / pairs * ca + (double)n * cb);
    }
    if (extra == std::max(0, most - 1) || time < best.time) {
      best.extra = extra;
      best.time = time;
    }
  }
  return best;
}

// The forward's tiles, wide or narrow, and the number of pairs.
inline Division divide_fwd(int64_t tokens, int64_t dim, int64_t hidden, int sms,
                           int* pairs) {
  Division d = {};
  d.kind[0] = d.kind[1] = kFwd;
  Shares best = {};
  for (int narrow = 0; narrow < 2; ++narrow) {
    const Tiles t = make_tiles(tokens, hidden, kHalf, 1, up(dim, kStep), narrow);
    const Shares s = share(t, d.tile[1], sms);
    if (narrow > 0 && s.time >= best.time) continue;
    best = s;
    d.tile[0] = t;
  }
  d.heavy = best.heavy;
  d.extra = best.extra;
  *pairs = best.pairs;
  return d;
}

// The backward's: the tiles with the longer sums first, each kind as wide as ends
// first.  Frozen weights have none.
inline Division divide_bwd(int64_t tokens, int64_t dim, int64_t hidden,
                           bool weights, int sms, int* pairs) {
  Division d = {};
  Shares best = {};
  for (int narrow = 0; narrow < 4; ++narrow) {
    const Tiles dx = make_tiles(tokens, dim, 2 * kHalf, 1, 2 * up(hidden, kStep),
                                narrow & 1);
    Tiles dw = make_tiles(hidden, dim, 2 * kHalf, 2, up(tokens, kStep),
                          narrow >> 1);
    if (!weights) dw.count = 0;
    const int first = weights && dw.steps > dx.steps ? 1 : 0;
    const Tiles& a = first ? dw : dx;
    const Tiles& b = first ? dx : dw;
    const Shares s = share(a, b, sms);
    if (narrow > 0 && s.time >= best.time) continue;
    best = s;
    d.tile[0] = a;
    d.tile[1] = b;
    d.kind[first] = kDx;
    d.kind[1 - first] = kDw;
  }
  d.heavy = best.heavy;
  d.extra = best.extra;
  *pairs = best.pairs;
  return d;
}

}  // namespace ffn
}  // namespace fastvr
