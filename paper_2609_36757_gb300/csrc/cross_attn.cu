// Cross attention forward on tcgen05 tensor cores: out = softmax(scale q k^T) v
// over the first kv_len[b] of kv_tokens keys, heads in groups that share a key
// head.
//
// Few keys (a prompt) and many queries: above some 300 keys the products are its
// floor, below that HBM (q in, out back), and a unit of work (two tiles of 128
// queries over all keys) is short.  So the kernel is
// persistent and its units follow one another without a gap: the schedule is
// chunk_attn_fwd.cu's (QK_0(j), PV_0(j-1), QK_1(j), PV_1(j-1), one S tile shared
// by both query tiles, PV one key tile behind), taken across the units' ends,
// where the queries of the next unit come from a ring of tiles and a tile's
// output leaves between its last PV and the next unit's first:
//   warp 8      TMA producer of the query and the K tiles (rings)
//   warp 10     TMA producer of the V tiles (ring)
//   warp 11     relay: hands landed tiles to the MMA warp through named barriers
//               and zeroes V rows past the last key (their contents, which may
//               be NaN, would meet P = 0)
//   warp 9      MMA issuer
//   warps 0-3, 4-7  softmax and output of the first and second query tile
// TMEM (512 columns): S | P_0 | P_1 | O_0 | O_1.
//
// With many keys it runs at the rate of chunk_attn_fwd.cu's steps (145 us for 19456
// tokens of 12 heads over 2048 keys, 1690 TFLOP/s; 8192 by 8192 of 57 heads 1880).
// With few, a unit's end counts: the output keeps a query tile's warps from their
// next scores (46.2 us over 512 keys, 41.0 without the stores; through shared memory
// and TMA stores, or by warps of their own, it was no faster).  The first copies
// take 3 to 4 us of a launch.  What the kernel is sensitive to is the MMA warp's
// issue (warp_uniform).  With entries of different lengths CTAs take ranges of
// query tiles of about equal work.
//
// P enters its product with V in bfloat16, as the tensor cores want both operands of
// one type; row sums take it unrounded.  Outputs are off by 2.3e-3 in the 2-norm, by
// 1.7e-3 from their own rounding alone.
//
// Waits on mbarriers are bounded; past the limit every role stops.  The MMA
// warp waits on named barriers, which have no limit: after a failure the relay
// keeps arriving on all of them until the MMA warp has left.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "attn_softmax.cuh"
#include "cross_attn.cuh"
#include "fastvr_internal.h"
#include "sm100_ptx.cuh"

namespace fastvr {
namespace {

using namespace sm100;

constexpr int kBM = 128;         // query rows per tile (one TMEM lane each)
constexpr int kBN = 128;         // keys per tile
constexpr int kThreads = 384;
constexpr int kBox = 128 * 128;  // one TMA box: 128 rows x 64 bf16 (bytes)
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kTmemS = 0, kTmemP = 128, kTmemO = 256;
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr uint64_t kDefaultWaitLimitNs = 4000000000ull;
// The relay keeps the MMA warp going for this and three waits: far longer than that
// warp needs to see a failure, since a named barrier has no limit.
constexpr uint64_t kReleaseNs = 1000000000ull;
// Named barriers of the hand-offs to the MMA warp.
constexpr int kBarSFree = 1;
constexpr int kBarP = 2;   // + query tile
constexpr int kBarK = 4;   // + stage (at most 3)
constexpr int kBarV = 7;   // + stage (at most 3)
constexpr int kBarQ = 10;  // + stage (at most 4)
constexpr int kBars = 14;
constexpr int kHandoff = 5 * 32;  // four softmax warps and the MMA warp
constexpr int kRelay = 2 * 32;

template <int D>
struct Layout {
  static constexpr int kNB = D / 64;  // boxes per tile
  static constexpr int kTile = kNB * kBox;
  static constexpr int kQ = D == 64 ? 4 : 3;  // ring stages
  static constexpr int kK = D == 64 ? 3 : 2;
  static constexpr int kV = D == 64 ? 3 : 2;
  static constexpr int k_off = kQ * kTile;
  static constexpr int v_off = k_off + kK * kTile;
  static constexpr int shared_off = v_off + kV * kTile;
  static constexpr int bytes = shared_off + 1024 /*Shared*/ + 1024 /*align*/;
};

struct CrossParams {
  CUtensorMap q_map, k_map, v_map;  // {d, tokens, heads, batch}
  uint16_t* o;
  float* lse;
  Strides o_str;
  const int32_t* kv_len;
  int32_t batch, heads, group, q_tokens, kv_tokens;
  int32_t q_tiles;          // of a head
  int32_t per_slot, slots;  // query tiles of a slot (1 or 2), slots of a head
  int32_t all, step;        // slots of all heads; from a CTA's slot to its next
  FastDiv by_slots, by_heads, by_group;
  int32_t q_batch, k_batch, v_batch;  // 0: one entry for the whole batch
  int32_t wide;                       // output rows on 32-byte boundaries
  float scale_log2;
  int* status;
  int32_t inject_stall;
  uint64_t wait_limit_ns;
};

struct Shared {
  uint64_t q_full[4], q_empty[4], k_full[3], k_empty[3], v_full[3], v_empty[3];
  uint64_t s_full[2], p_free[2], drain;
  uint32_t tmem_base;
  int abort, mma_done;
  int first, last;  // the CTA's slots: first, first + step, ... below last
  uint64_t wait_limit_ns;
};
static_assert(sizeof(Shared) <= 1024, "Shared fits its place");

// A unit: two tiles of one (b, h)'s queries (or one, at an end) over its keys.
struct Unit {
  int b, h, q0, len, n;  // n: key tiles
  bool two;
};
// The unit at slot x; returns the slot behind it.  Slots are pairs of query
// tiles, or single ones, two neighbours of a CTA then making a unit.
__device__ __forceinline__ int get_unit(const CrossParams& p, int x, int last,
                                        Unit* u) {
  const uint32_t bh = fast_div(x, p.by_slots);
  const int t = (int)(x - bh * p.slots) * p.per_slot;
  u->q0 = t * kBM;
  u->b = (int)fast_div(bh, p.by_heads);
  u->h = (int)(bh - (uint32_t)u->b * p.heads);
  u->two = t + 1 < p.q_tiles && (p.per_slot == 2 || x + 1 < last);
  u->len = cross_keys(p.kv_len, u->b, p.kv_tokens);
  u->n = (u->len + kBN - 1) / kBN;
  return x + (p.per_slot == 1 ? 1 + (int)u->two : p.step);
}
// The CTA's next unit that has keys, from x on; false when there is none.
__device__ __forceinline__ bool next_unit(const CrossParams& p, int& x, int last,
                                          Unit* u) {
  while (x < last) {
    x = get_unit(p, x, last, u);
    if (u->n > 0) return true;
  }
  return false;
}
// First slot of CTA c: of about equal work to each, a slot weighing its key tiles
// and one more for its way in and out (of equal numbers, for batches so large that
// the sums would take longer than they save).  A whole warp's.
constexpr int kMaxWeighed = 4096;
__device__ __forceinline__ int first_slot(const CrossParams& p, int c,
                                          int lane) {
  if (p.step > 1) return c;
  if (p.kv_len == nullptr || p.batch > kMaxWeighed || c == (int)gridDim.x)
    return (int)((int64_t)p.all * c / gridDim.x);
  const int per = p.heads * p.slots;  // of a batch entry
  const int chunk = (p.batch + 31) / 32;
  const int b0 = min(lane * chunk, p.batch), b1 = min(b0 + chunk, p.batch);
  auto weight = [&](int b) {
    return 1 + (cross_keys(p.kv_len, b, p.kv_tokens) + kBN - 1) / kBN;
  };
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += weight(b);
  int64_t before = mine;  // of the lanes before this one, and of all
  for (int d = 1; d < 32; d *= 2) {
    const int64_t x = __shfl_up_sync(~0u, before, d);
    if (lane >= d) before += x;
  }
  const int64_t total = __shfl_sync(~0u, before, 31);
  before -= mine;
  // in units of a batch entry's tiles: position total * c / grid
  const int64_t num = total * c;  // / gridDim.x
  int found = -1;
  int64_t at = before * gridDim.x;
  for (int b = b0; b < b1 && found < 0; ++b) {
    const int64_t w = (int64_t)weight(b) * gridDim.x;
    if (num < at + w)
      found = num >= at ? b * per + (int)((double)(num - at) / (double)w * per)
                        : -2;
    at += w;
  }
  found = max(found, 0);
  for (int d = 16; d > 0; d /= 2)
    found = max(found, __shfl_xor_sync(~0u, found, d));
  return min(found, p.all);
}

__device__ __forceinline__ bool give_up(Shared* S, uint64_t t0, int* status) {
  if (*reinterpret_cast<volatile int*>(&S->abort)) return true;
  if (global_timer_ns() - t0 <= S->wait_limit_ns) return false;
  *reinterpret_cast<volatile int*>(&S->abort) = 1;
  if (status != nullptr) atomicExch(status, kDevTimeout);
  return true;
}
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity,
                                         Shared* S, int* status) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity))
    if (give_up(S, t0, status)) return false;
  return true;
}
// The whole warp's, which stays converged.
__device__ __forceinline__ bool wait_bar_warp(uint64_t* bar, uint32_t parity,
                                              Shared* S, int* status) {
  if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
  const uint64_t t0 = global_timer_ns();
  while (!__all_sync(~0u, mbar_try_wait(bar, parity)))
    if (__any_sync(~0u, give_up(S, t0, status))) return false;
  return true;
}
// Ignores the abort flag (draining what is in flight).
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity,
                                           const Shared* S) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity))
    if (global_timer_ns() - t0 > S->wait_limit_ns) return;
}

__device__ __forceinline__ void handoff_arrive(int id) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kHandoff) : "memory");
}
__device__ __forceinline__ void handoff_sync(int id) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kHandoff) : "memory");
}
__device__ __forceinline__ void relay_arrive(int id) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kRelay) : "memory");
}
__device__ __forceinline__ void relay_sync(int id) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kRelay) : "memory");
}

// The first query tile, K_0, the second query tile, K_1, ...: the order in which
// the MMA warp takes them.
template <int D>
__device__ void qk_producer(const CrossParams& p, uint8_t* smem, Shared* S) {
  using L = Layout<D>;
  // a query tile is read once, the keys of a head by every unit of it
  const uint64_t once = l2_policy_evict_first(), keep = l2_policy_evict_last();
  const int end = S->last;
  int x = S->first, qc = 0, kc = 0;
  Unit u;
  bool ok = true;
  while (ok && next_unit(p, x, end, &u)) {
    const int hk = (int)fast_div(u.h, p.by_group);
    auto query = [&](int t) {
      const int st = qc % L::kQ;
      if (!(ok = wait_bar(&S->q_empty[st], ((qc / L::kQ) & 1) ^ 1, S,
                          p.status)))
        return;
      mbar_arrive_expect_tx(&S->q_full[st], L::kTile);
      for (int bx = 0; bx < L::kNB; ++bx)
        tma_load_4d_hint(&p.q_map, smem + st * L::kTile + bx * kBox,
                         &S->q_full[st], bx * 64, u.q0 + t * kBM, u.h,
                         u.b * p.q_batch, once);
      ++qc;
    };
    query(0);
    for (int j = 0; ok && j < u.n; ++j) {
      const int st = kc % L::kK;
      if (!(ok = wait_bar(&S->k_empty[st], ((kc / L::kK) & 1) ^ 1, S,
                          p.status)))
        break;
      mbar_arrive_expect_tx(&S->k_full[st], L::kTile);
      for (int bx = 0; bx < L::kNB; ++bx)
        tma_load_4d_hint(&p.k_map, smem + L::k_off + st * L::kTile + bx * kBox,
                         &S->k_full[st], bx * 64, j * kBN, hk,
                         u.b * p.k_batch, keep);
      ++kc;
      if (j == 0 && u.two) query(1);
    }
  }
  // every load has landed before the CTA exits
  for (int i = max(0, qc - L::kQ); i < qc; ++i)
    drain_wait(&S->q_full[i % L::kQ], (i / L::kQ) & 1, S);
  for (int i = max(0, kc - L::kK); i < kc; ++i)
    drain_wait(&S->k_full[i % L::kK], (i / L::kK) & 1, S);
}

template <int D>
__device__ void v_producer(const CrossParams& p, uint8_t* smem, Shared* S) {
  using L = Layout<D>;
  const uint64_t keep = l2_policy_evict_last();
  const int end = S->last;
  int x = S->first, vc = 0;
  Unit u;
  // Test hook: the others' waits run out too, the MMA warp amid a unit.
  bool ok = p.inject_stall != 2 || wait_bar(&S->drain, 0, S, p.status);
  while (ok && next_unit(p, x, end, &u)) {
    const int hk = (int)fast_div(u.h, p.by_group);
    for (int j = 0; j < u.n; ++j) {
      const int st = vc % L::kV;
      if (!(ok = wait_bar(&S->v_empty[st], ((vc / L::kV) & 1) ^ 1, S,
                          p.status)))
        break;
      mbar_arrive_expect_tx(&S->v_full[st], L::kTile);
      for (int bx = 0; bx < L::kNB; ++bx)
        tma_load_4d_hint(&p.v_map, smem + L::v_off + st * L::kTile + bx * kBox,
                         &S->v_full[st], bx * 64, j * kBN, hk,
                         u.b * p.v_batch, keep);
      ++vc;
    }
  }
  for (int i = max(0, vc - L::kV); i < vc; ++i)
    drain_wait(&S->v_full[i % L::kV], (i / L::kV) & 1, S);
}

// Observes the landed tiles in the order in which the MMA warp takes them.
template <int D>
__device__ void relay_role(const CrossParams& p, uint8_t* smem, Shared* S,
                           int lane) {
  using L = Layout<D>;
  const int end = S->last;
  int x = S->first, qc = 0, kc = 0, vc = 0;
  Unit u;
  bool ok = true, pend = false, have = next_unit(p, x, end, &u);
  int j = 0, pvalid = 0;
  auto query = [&]() {
    const int st = qc % L::kQ;
    if ((ok = ok && wait_bar_warp(&S->q_full[st], (qc / L::kQ) & 1, S,
                                  p.status)))
      relay_arrive(kBarQ + st);
    ++qc;
  };
  while (ok && (have || pend)) {
    if (have) {
      if (j == 0) query();
      const int st = kc % L::kK;
      if ((ok = ok && wait_bar_warp(&S->k_full[st], (kc / L::kK) & 1, S,
                                    p.status)))
        relay_arrive(kBarK + st);
      ++kc;
    }
    if (ok && pend) {
      const int st = vc % L::kV;
      if ((ok = wait_bar_warp(&S->v_full[st], (vc / L::kV) & 1, S,
                              p.status))) {
        // A row is 128 bytes of each box; the swizzle stays within rows.  Without
        // lengths the rows past the last key lie outside the map: zeros.
        if (pvalid < kBN && p.kv_len != nullptr) {
          for (int bx = 0; bx < L::kNB; ++bx) {
            uint4* rows = reinterpret_cast<uint4*>(smem + L::v_off +
                                                   st * L::kTile + bx * kBox);
            for (int i = pvalid * 8 + lane; i < kBN * 8; i += 32)
              rows[i] = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        relay_arrive(kBarV + st);
      }
      ++vc;
    }
    if (ok && have && j == 0 && u.two) query();
    pend = have;
    if (have) {
      pvalid = min(kBN, u.len - j * kBN);
      if (++j == u.n) {
        j = 0;
        have = next_unit(p, x, end, &u);
      }
    }
  }
  // The MMA warp may still wait for arrivals that a failed role will not make.
  volatile int* done = &S->mma_done;
  volatile int* abort = &S->abort;
  const uint64_t t0 = global_timer_ns();
  while (!__any_sync(~0u, *done != 0)) {
    if (__any_sync(~0u, *abort != 0)) {
      for (int id = kBarSFree; id < kBarK; ++id) handoff_arrive(id);
      for (int id = kBarK; id < kBars; ++id) relay_arrive(id);
    }
    if (__any_sync(~0u, global_timer_ns() - t0 >
                            3 * S->wait_limit_ns + kReleaseNs))
      break;
    __nanosleep(200);
  }
}

__device__ __forceinline__ uint32_t read_abort(const Shared* S) {
  uint32_t a;
  asm volatile("ld.volatile.shared.u32 %0, [%1];"
               : "=r"(a)
               : "r"(smem_addr(&S->abort)));
  return a;
}

// The MMA warp stops within twice this many key tiles of a failure, each of which
// takes a few rounds of the relay's arrivals: a millisecond or two in all.
constexpr int kIssue = 128;
template <int D>
__device__ void mma_issuer(const CrossParams& p, uint8_t* smem, Shared* S,
                           uint32_t tmem) {
  using L = Layout<D>;
  constexpr uint32_t kIdescQK = idesc_bf16_f32(kBM, kBN, 0);
  constexpr uint32_t kIdescPV = idesc_bf16_f32(kBM, D, 1);
  // Both query tiles' part of a step is unrolled, but for heads of 64, whose MMAs
  // are half as long, fetching the code takes longer than is saved (67.9 us for
  // 19456 tokens of 24 heads over 512 keys, unrolled 69.2).
  constexpr int kSides = D == 64 ? 1 : 2;
  const uint32_t sbase = smem_addr(smem);
  const uint32_t hi = desc_hi_sw128(1024);
  const uint32_t q_lo = desc_lo(sbase, 16);
  const uint32_t k_lo = desc_lo(sbase + L::k_off, 16);
  const uint32_t v_lo = desc_lo(sbase + L::v_off, kBox);
  constexpr uint32_t kStage16 = (uint32_t)L::kTile >> 4;
  auto qk = [&](uint32_t a0, uint32_t b0) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const uint32_t off = (uint32_t)((ks / 4) * kBox + (ks % 4) * 32) >> 4;
      mma_ss_warp(tmem + kTmemS, a0 + off, b0 + off, hi, kIdescQK, ks > 0);
    }
  };
  auto pv = [&](int t, uint32_t b0, bool acc) {
#pragma unroll
    for (int kk = 0; kk < kBN / 16; ++kk)
      mma_ts_warp(tmem + kTmemO + t * 128, tmem + kTmemP + t * 64 + kk * 8,
                  b0 + (uint32_t)(kk * 2048 >> 4), hi, kIdescPV,
                  acc || kk > 0);
  };
  auto take_s = [&](bool wait) {
    if (wait) handoff_sync(kBarSFree);
    tc_fence_after();
  };
  // Test hook: `drain` receives no arrival before the end, so this wait runs
  // out and exercises the abort path.
  bool ok = p.inject_stall != 1 || wait_bar_warp(&S->drain, 0, S, p.status);
  const int end = warp_uniform(S->last);
  int x = warp_uniform(S->first);
  int s = 0, qc = 0;  // steps and query tiles so far
  bool ptwo = false, pacc = false;  // of the step whose PV is owed
  // PV_t of step i.
  auto owed = [&](int t, int i, bool two) {
    const int vs = i % L::kV;
    if (t == 0) relay_sync(kBarV + vs);
    handoff_sync(kBarP + t);
    tc_fence_after();
    pv(t, v_lo + vs * kStage16, pacc);
    mma_commit_warp(&S->p_free[t]);
    if (t == (int)two) mma_commit_warp(&S->v_empty[vs]);
  };
  Unit u;
  while (warp_uniform(ok && next_unit(p, x, end, &u))) {
    const int n = warp_uniform(u.n);
    const bool two = warp_uniform(u.two);
    x = warp_uniform(x);
    const int q0 = qc % L::kQ, q1 = (qc + 1) % L::kQ;
    qc += 1 + (int)two;
    for (int j = 0; ok && j < n;) {
      const uint32_t aborted = read_abort(S);  // looked at kIssue steps later
      const int stop = min(n, j + kIssue);
      for (; j < stop; ++j, ++s) {
        const int ks = s % L::kK;
#pragma unroll kSides
        for (int t = 0; t < 2; ++t) {
          if (t <= (int)two) {
            const int q = t == 0 ? q0 : q1;
            if (j == 0) relay_sync(kBarQ + q);
            if (t == 0) relay_sync(kBarK + ks);
            take_s(s + t > 0);
            qk(q_lo + q * kStage16, k_lo + ks * kStage16);
            mma_commit_warp(&S->s_full[t]);
            if (j == n - 1) mma_commit_warp(&S->q_empty[q]);
            if (t == (int)two) mma_commit_warp(&S->k_empty[ks]);
          }
          if (s > 0 && t <= (int)ptwo) owed(t, s - 1, ptwo);
        }
        ptwo = two;
        pacc = j > 0;
      }
      if (__any_sync(~0u, aborted != 0)) ok = false;
    }
  }
  if (ok && s > 0) {
#pragma unroll 1
    for (int t = 0; t <= (int)ptwo; ++t) owed(t, s - 1, ptwo);
  }
  mma_commit_warp(&S->drain);
  if ((threadIdx.x & 31) == 0) {
    drain_wait(&S->drain, 0, S);
    *reinterpret_cast<volatile int*>(&S->mma_done) = 1;
  }
  __syncwarp();
}

// out = O / l from TMEM, where a lane has a row.  With heads of 128 lanes 2 i and
// 2 i + 1 exchange pieces of 32 bytes (whole sectors), so that a store writes 64 bytes
// of 16 rows, `first` being the even lane's row and `second` the odd one's, instead of
// 32 bytes of 32 rows: 43.0 us instead of 45.8 for the 1080p chunk, 18.9 instead of 19.9
// for 7440 tokens over 226 keys; 12.1 instead of 11.8 for 3180, two short units to a CTA,
// the one of seven sizes that loses more than a hundredth.  A row of 64 has
// too few of them (67.9 us for 19456 tokens of 24 heads over 512 keys, 73.4 with the
// exchange): `first` is the lane's own.
template <int D>
__device__ __forceinline__ void write_rows(uint16_t* first,
                                           uint16_t* second, int lane,
                                           uint32_t tO, float l, bool wide) {
  const float inv = 1.f / l;
  const bool b = lane & 1;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    uint32_t v[32], pk[16];
    __syncwarp();
    tmem_ld32(tO + c * 32, v);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i)
      pk[i] = pack_bf16(__uint_as_float(v[2 * i]) * inv,
                        __uint_as_float(v[2 * i + 1]) * inv);
    if (D == 64) {
      if (first != nullptr) {
        store_piece(first + c * 32, pk, wide);
        store_piece(first + c * 32 + 16, pk + 8, wide);
      }
    } else {
      swap_pieces(pk, b);
      const int at = c * 32 + 16 * b;
      if (first != nullptr) store_piece(first + at, pk, wide);
      if (second != nullptr) store_piece(second + at, pk + 8, wide);
    }
  }
  __syncwarp();
}

constexpr int kLook = 1024;
template <int D>
__device__ void softmax_role(const CrossParams& p, Shared* S, uint32_t tmem,
                             int t, int wq, int lane) {
  const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
  const uint32_t tS = tmem + kTmemS + lane_off;
  const uint32_t tP = tmem + kTmemP + t * 64 + lane_off;
  const uint32_t tO = tmem + kTmemO + t * 128 + lane_off;
  const int r = wq * 32 + lane;  // row within the tile
  const float sl2 = p.scale_log2;
  const uint64_t sl2x2 = f2_pack(sl2, sl2);
  // With heads of 128 the loop over units has no registers to spare for uniform
  // control flow (50.7 us over 512 keys instead of 49.2); with 64 it takes 68.6 us
  // instead of 80.7.
  auto uniform = [](int v) { return D == 64 ? warp_uniform(v) : v; };
  const int end = uniform(S->last);
  int tiles = 0;  // key tiles of this query tile so far: barrier phases
  // the slot of the unit whose output is owed (-1: none), the row's sum
  int owed = -1;
  float owed_l = 0.f;
  bool ok = true;
  // A row's places in out and lse; computed anew where they are needed, since
  // the loop over the keys has no registers to hold them.
  auto out_row = [&](const Unit& u, int row) {
    return p.o + (int64_t)u.b * p.o_str.batch +
           (int64_t)(u.q0 + t * kBM + row) * p.o_str.token +
           (int64_t)u.h * p.o_str.head;
  };
  auto lse_row = [&](const Unit& u) {
    return p.lse + ((int64_t)u.b * p.heads + u.h) * p.q_tokens + u.q0 +
           t * kBM + r;
  };
  auto exists = [&](const Unit& u, int row) {
    return u.q0 + t * kBM + row < p.q_tokens && (t == 0 || u.two);
  };
  auto write_owed = [&]() {
    Unit u;
    get_unit(p, owed, end, &u);
    const int x = D == 64 ? r : r & ~1;
    write_rows<D>(
        exists(u, x) ? out_row(u, x) : nullptr,
        D == 128 && exists(u, x + 1) ? out_row(u, x + 1) : nullptr, lane, tO,
        owed_l, p.wide);
  };
  for (int slot = uniform(S->first), next; uniform(ok && slot < end);
       slot = next) {
    int n, len;
    bool unfollowed;  // no QK^T follows this unit's last S of this tile
    {
      Unit u, v;
      next = uniform(get_unit(p, slot, end, &u));
      n = warp_uniform(u.n);
      len = warp_uniform(u.len);
      if (n == 0) {  // sees no key
        if (exists(u, r)) {
          for (int c = 0; c < D; c += 8)
            *reinterpret_cast<uint4*>(out_row(u, r) + c) = make_uint4(0, 0, 0, 0);
          if (p.lse != nullptr) *lse_row(u) = -INFINITY;
        }
        __syncwarp();
        continue;
      }
      if (t == 1 && !u.two) continue;
      int y = next;
      unfollowed = t == (int)u.two && !next_unit(p, y, end, &v);
    }
    float m_ref = -INFINITY, l = 0.f;
    // A wait may run out for some lanes of a warp and end well for others, so none
    // leaves alone: the warp meets again, as the accesses to TMEM and the named
    // barriers ask for, goes on, and looks at the abort flag together, every kLook
    // tiles (a vote on every wait took 46.9 us for the 1080p chunk instead of 45.8).
    for (int j = 0; ok && j < n;) {
      const int stop = min(n, j + kLook);
      const bool ends = unfollowed && stop == n;
      for (; j < stop; ++j) {
        wait_bar(&S->s_full[t], tiles & 1, S, p.status);
        __syncwarp();
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(tS + 32 * c, s[c]);
        tmem_wait_ld();
        tc_fence_before();
        // no QK^T follows the CTA's last S
        if (!ends || j < stop - 1) handoff_arrive(kBarSFree);
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        const int valid = len - j * kBN;
#pragma unroll
        for (int c = 0; c < 4; ++c) mask_max32(s[c], c, valid, mx);
        const float mrow = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * sl2;
        const bool rescale =
            __any_sync(~0u, mrow > m_ref + kRescaleThreshold);
        float alpha = 1.f;
        if (rescale) {
          const float m_new = fmaxf(m_ref, mrow);
          alpha = m_ref == -INFINITY ? 0.f : ex2(m_ref - m_new);
          l *= alpha;
          m_ref = m_new;
        }
        // a row whose scores are all -infinity so far exponentiates against 0
        const float neg = m_ref == -INFINITY ? 0.f : -m_ref;
        const uint64_t neg2 = f2_pack(neg, neg);
        uint64_t acc[4] = {0, 0, 0, 0};
        uint32_t pk[2][16];
#pragma unroll
        for (int c = 0; c < 2; ++c) exp_pack32(s[c], sl2x2, neg2, pk[c], acc);
        // this query tile's previous PV is done: P may be written, O is current
        if (tiles > 0) wait_bar(&S->p_free[t], (tiles - 1) & 1, S, p.status);
        __syncwarp();
        tc_fence_after();
        if (j == 0) {
          if (owed >= 0) write_owed();
        } else if (rescale) {
#pragma unroll 1
          for (int c = 0; c < D / 8; ++c) {
            uint32_t v[8];
            tmem_ld8(tO + c * 8, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
            tmem_st8(tO + c * 8, v);
          }
        }
        tmem_st16(tP, pk[0]);
        tmem_st16(tP + 16, pk[1]);
#pragma unroll
        for (int c = 2; c < 4; ++c) {
          exp_pack32(s[c], sl2x2, neg2, pk[c - 2], acc);
          tmem_st16(tP + 16 * c, pk[c - 2]);
        }
        l += acc_total(acc);
        tmem_wait_st();
        tc_fence_before();
        handoff_arrive(kBarP + t);
        ++tiles;
      }
      ok = !__any_sync(~0u, read_abort(S));
    }
    if (!ok) break;
    Unit u;
    get_unit(p, slot, end, &u);
    if (exists(u, r) && p.lse != nullptr)
      *lse_row(u) = (m_ref + __log2f(l)) * 0.6931471805599453f;
    owed = slot;
    owed_l = l;
  }
  if (ok && owed >= 0 &&
      wait_bar_warp(&S->p_free[t], (tiles - 1) & 1, S, p.status)) {
    tc_fence_after();
    write_owed();
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
cross_tile_kernel(const __grid_constant__ CrossParams p) {
  using L = Layout<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Shared* S = reinterpret_cast<Shared*>(smem + L::shared_off);
  const int warp = warp_uniform(threadIdx.x / 32);
  const int lane = threadIdx.x % 32;
  if (warp == 9) {
    tmem_alloc(&S->tmem_base, kTmemCols);
    tmem_relinquish();
  }
  if (threadIdx.x == 320) {
    tma_prefetch_desc(&p.q_map);
    tma_prefetch_desc(&p.k_map);
    tma_prefetch_desc(&p.v_map);
  }
  if (threadIdx.x == 256) {
    for (int s = 0; s < L::kQ; ++s) {
      mbar_init(&S->q_full[s], 1);
      mbar_init(&S->q_empty[s], 1);
    }
    for (int s = 0; s < L::kK; ++s) {
      mbar_init(&S->k_full[s], 1);
      mbar_init(&S->k_empty[s], 1);
    }
    for (int s = 0; s < L::kV; ++s) {
      mbar_init(&S->v_full[s], 1);
      mbar_init(&S->v_empty[s], 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&S->s_full[t], 1);
      mbar_init(&S->p_free[t], 1);
    }
    mbar_init(&S->drain, 1);
    S->abort = 0;
    S->mma_done = 0;
    S->wait_limit_ns = p.wait_limit_ns ? p.wait_limit_ns : kDefaultWaitLimitNs;
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(S->tmem_base);
  pdl_trigger();
  pdl_wait();
  if (warp < 2) {
    const int at = warp == 1 && p.step > 1
                       ? p.all
                       : first_slot(p, blockIdx.x + warp, lane);
    if (lane == 0) (warp == 0 ? S->first : S->last) = at;
  }
  __syncthreads();

  if (warp == 8) {
    if (lane == 0) qk_producer<D>(p, smem, S);
    __syncwarp();
  } else if (warp == 10) {
    if (lane == 0) v_producer<D>(p, smem, S);
    __syncwarp();
  } else if (warp == 9) {
    mma_issuer<D>(p, smem, S, tmem);
  } else if (warp == 11) {
    relay_role<D>(p, smem, S, lane);
  } else {
    softmax_role<D>(p, S, tmem, warp / 4, warp % 4, lane);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int D>
cudaError_t launch_tiles(const CrossArgs& a, cudaStream_t stream) {
  CrossParams p;
  memset(&p, 0, sizeof(p));
  if (!cross_map(&p.q_map, a.q, D, a.q_tokens, a.heads, a.batch, a.q_str,
                 &p.q_batch) ||
      !cross_map(&p.k_map, a.k, D, a.kv_tokens, a.kv_heads, a.batch, a.k_str,
                 &p.k_batch) ||
      !cross_map(&p.v_map, a.v, D, a.kv_tokens, a.kv_heads, a.batch, a.v_str,
                 &p.v_batch))
    return cudaErrorInvalidValue;
  p.o = a.o;
  p.lse = a.lse;
  p.o_str = a.o_str;
  p.kv_len = a.kv_len;
  p.batch = a.batch;
  p.heads = a.heads;
  p.group = a.heads / a.kv_heads;
  p.q_tokens = a.q_tokens;
  p.kv_tokens = a.kv_tokens;
  p.q_tiles = (a.q_tokens + kBM - 1) / kBM;
  // Pairs unless they leave some CTA more units than single tiles would (25 tiles
  // of each of 12 heads over 152 CTAs: 156 pairs, but two tiles to each).
  const int heads = a.batch * a.heads;
  const int pairs = (p.q_tiles + 1) / 2;
  auto each = [&](int n) { return (n * heads + a.sms - 1) / a.sms; };
  const bool paired = each(pairs) <= (each(p.q_tiles) + 1) / 2 &&
                      p.q_tiles * heads > a.sms;
  p.per_slot = paired ? 2 : 1;
  p.slots = paired ? pairs : p.q_tiles;
  p.all = p.slots * heads;
  p.by_slots = make_div((uint32_t)p.slots);
  const int grid = std::min(p.all, a.sms);
  // Pairs of equal work are dealt out in turn, so that the last ones run with the
  // GPU to themselves; others are taken in ranges of equal work.
  p.step = paired && a.kv_len == nullptr ? grid : 1;
  p.by_heads = make_div((uint32_t)a.heads);
  p.by_group = make_div((uint32_t)p.group);
  p.wide = ((uintptr_t)a.o & 31) == 0 && a.o_str.batch % 16 == 0 &&
           a.o_str.token % 16 == 0 && a.o_str.head % 16 == 0;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.status = a.status;
  p.inject_stall = a.inject_stall;
  p.wait_limit_ns = a.wait_limit_ns;
  const int smem = Layout<D>::bytes;
  static_assert(Layout<D>::bytes <= 227 * 1024, "shared memory");
  const cudaError_t e = allow_smem<cross_tile_kernel<D>>(smem, a.device);
  if (e != cudaSuccess) return e;
  return launch_pdl(cross_tile_kernel<D>, dim3(grid),
                    dim3(kThreads), smem, stream, p);
}

}  // namespace

// A [batch, tokens, heads, d] tensor as a map over (d, token, head, batch), box
// 64 x 128.  The stride of a dimension of one entry does not matter; a batch
// stride of 0 becomes a batch of one, *batch_step 0.
bool cross_map(CUtensorMap* m, const void* base, int d, int tokens, int heads,
               int batch, const Strides& str, int32_t* batch_step) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (enc == nullptr) return false;
  *batch_step = batch > 1 && str.batch > 0;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)tokens,
                              (cuuint64_t)heads,
                              (cuuint64_t)(*batch_step ? batch : 1)};
  const int64_t given[3] = {str.token, str.head, str.batch};
  cuuint64_t strides[3];
  for (int i = 0; i < 3; ++i)
    strides[i] = (cuuint64_t)(dims[i + 1] > 1 ? given[i] : d) * 2;
  const cuuint32_t box[4] = {64, 128, 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base),
             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_cross_attn(const CrossArgs& a, cudaStream_t stream) {
  if (cross_few_rows((int64_t)a.q_tokens * (a.heads / a.kv_heads)))
    return launch_cross_rows(a, stream);
  return a.head_dim == 64 ? launch_tiles<64>(a, stream)
                          : launch_tiles<128>(a, stream);
}

}  // namespace fastvr
