// Cross attention backward on tcgen05 tensor cores.
//
// With P = softmax(scale q k^T), recomputed from the forward's log-sum-exp, and
// D_i = <dO_i, O_i>:
//     dV = P^T dO,  dP = dO V^T,  dS = P o (dP - D),
//     dQ = scale dS K,  dK = scale dS^T Q,
// dK and dV summed over the query heads that share a key head.  As in
// chunk_attn_bwd.cu, without atomics, in kernels that each keep their results in
// TMEM:
//   rows_kernel   D_i and the log-sum-exp in log2 units, both negated, one
//                 padded row of scratch per (b, h);
//   grads_kernel  both of these at once, so that each fills the SMs that the other's
//                 last CTAs leave idle:
//   dkdv_cta      one CTA per tile of 128 keys and range of query tiles (of all
//                 heads of the group): S^T = K Q^T, dP^T = V dO^T, dV += P^T dO,
//                 dK += dS^T Q.  Keys are few and queries many, so a key tile's
//                 queries are cut into as many ranges as fill the GPU, whose
//                 float32 sums join_kernel adds up in order;
//   dq_cta        a CTA takes a few units, a unit being a tile of 128 queries over all keys of
//                 its head: S = Q K^T, dP = dO V^T, dQ += dS K.  With few keys a
//                 unit is short, so units follow one another without a gap: the
//                 next unit's S and dP run before this one's last dQ, whose
//                 result leaves between the next unit's P and dS.
// Measured at 12288 tokens of 24 heads of 128 over 512 keys: rows_kernel 27 us
// (O and dO at 5.6 TB/s), grads_kernel 182 (seven products of which dq's recompute
// two; 64 % of the tensor pipe's cycles: a unit of dq has four steps between its
// ends), join_kernel 10.
//
// P for dV, and dS (from the unrounded P), enter their products in bfloat16, the other
// operand's type, and D takes the forward's out as it was rounded, since no other is
// kept: gradients are off by 2.3e-3 to 2.6e-3 in the 2-norm (1.7e-3 from their own
// rounding), dQ and dK by up to 4.0e-3 with two to nine keys, where dP - D cancels.
//
// Lanes of TMEM are independent, so key rows past an entry's last need no mask
// in dkdv_cta (their results are replaced by zeros); in dq_cta their
// columns are masked and the K and V rows zeroed in shared memory, where NaN
// would meet P = 0.  Waits are bounded as in cross_attn.cu.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "attn_grad.cuh"
#include "cross_attn.cuh"
#include "fastvr_internal.h"
#include "sm100_ptx.cuh"

namespace fastvr {
namespace {

using namespace sm100;
using grad::exp2_poly;
using grad::f2;
using grad::f2_add;
using grad::f2_fma;
using grad::f2_mul;
using grad::f2_split;
using grad::pack_bf16;

constexpr int kT = 128;          // tile rows (TMEM lanes) and columns
constexpr int kBox = 128 * 128;  // one TMA box: 128 rows x 64 bf16 (bytes)
constexpr int kThreads = 384;
constexpr uint32_t kTmemCols = 512;
constexpr uint64_t kDefaultWaitLimitNs = 4000000000ull;
constexpr uint64_t kReleaseNs = 1000000000ull;  // cross_attn.cu
constexpr int kWarpA = 8, kMmaWarp = 9, kWarpB = 10, kRelayWarp = 11;
// Named barriers of the hand-offs to the MMA warp.  dq's dS has one for even and
// one for odd steps: its next S and dP are issued before the MMA warp waits for
// this dS, so a compute warp may hand over the next one while another still works
// on this one, and two arrivals of one warp would stand for both.
constexpr int kBarP = 1, kBarDS = 2;
constexpr int kBarRing = 4;  // + ring's first + stage
constexpr int kBars = 15;
constexpr int kComputeHandoff = 9 * 32;
constexpr int kRelayHandoff = 2 * 32;

struct BwdParams {
  CUtensorMap q_map, k_map, v_map, do_map;  // {d, tokens, heads, batch}
  const float* lse2;   // -(log-sum-exp in log2 units) [batch heads, padded]
  const float* delta;  // -D
  uint16_t *dq, *dk, *dv;
  Strides dq_str, dk_str, dv_str;
  const int32_t* kv_len;
  int32_t batch, heads, kv_heads, group, q_tokens, kv_tokens;
  int32_t padded, q_tiles, k_tiles, units;
  FastDiv by_q_tiles, by_heads, by_group;
  int32_t q_batch, k_batch, v_batch, do_batch;
  int32_t wide_q, wide_k, wide_v;
  int32_t parts;     // ranges of a key tile's query tiles
  int32_t dkdv_ctas, dq_ctas;
  float *dk_part, *dv_part;  // [parts][batch kv_heads][k_tiles * 128][d]
  float scale, scale_log2;
  int* status;
  int32_t inject_stall;
  uint64_t wait_limit_ns;
};

// A ring of tiles: barriers in Shared::full/empty from `first`, named barriers
// from kBarRing + first, `depth` stages at byte `off`.
template <int kFirst, int kDepth, int kOff>
struct Ring {
  static constexpr int first = kFirst, depth = kDepth, off = kOff;
};
constexpr int kRingSlots = 11;

struct Shared {
  uint64_t full[kRingSlots], empty[kRingSlots];
  uint64_t fixed_full, s_ready, dp_ready[2], out_full, drain;
  uint64_t vec_full[2], vec_empty[2];
  uint32_t tmem_base;
  int abort, mma_done;
  uint64_t wait_limit_ns;
};

// A front region with the barriers (and, for dK and dV, two slots of row vectors),
// then the tiles: 227 KB exactly at d = 128.
constexpr int kFront = 3 * 1024;

template <int D>
struct DqLayout {
  static constexpr int kNB = D / 64, kTile = kNB * kBox;
  // d = 128: seven tiles of 32 KB.  K needs three (K_j lives until dQ_j, two
  // products after S_{j+1}), V two.
  static constexpr int kPrev = D == 64 ? 2 : 1;
  using Q = Ring<0, kPrev, kFront>;
  using O = Ring<2, kPrev, kFront + kPrev * kTile>;
  using K = Ring<4, 3, kFront + 2 * kPrev * kTile>;
  using V = Ring<7, 2, kFront + (2 * kPrev + 3) * kTile>;
  static constexpr int bytes = kFront + (2 * kPrev + 5) * kTile;
};

// The resident K and V tiles, then the rings of Q and dO.
template <int D>
struct DkdvLayout {
  static constexpr int kNB = D / 64, kTile = kNB * kBox;
  __host__ __device__ static constexpr int vec(int slot, int which) {
    return 1024 + (slot * 2 + which) * kT * (int)sizeof(float);
  }
  static constexpr int k_off = kFront, v_off = kFront + kTile;
  using Q = Ring<0, 3, kFront + 2 * kTile>;
  using O = Ring<4, 2, kFront + 5 * kTile>;
  static constexpr int bytes = kFront + 7 * kTile;
};
static_assert(sizeof(Shared) <= 1024, "barriers fit their place");

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
__device__ __forceinline__ bool wait_bar_warp(uint64_t* bar, uint32_t parity,
                                              Shared* S, int* status) {
  if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
  const uint64_t t0 = global_timer_ns();
  while (!__all_sync(~0u, mbar_try_wait(bar, parity)))
    if (__any_sync(~0u, give_up(S, t0, status))) return false;
  return true;
}
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity,
                                           const Shared* S) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity))
    if (global_timer_ns() - t0 > S->wait_limit_ns) return;
}

__device__ __forceinline__ void compute_arrive(int id) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kComputeHandoff) : "memory");
}
__device__ __forceinline__ void compute_sync(int id) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kComputeHandoff) : "memory");
}
__device__ __forceinline__ void relay_arrive(int id) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kRelayHandoff) : "memory");
}
__device__ __forceinline__ void relay_sync(int id) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kRelayHandoff) : "memory");
}

// One tile into the ring's stage of its `count`-th tile.
template <int D, class R>
__device__ __forceinline__ bool ring_load(const BwdParams& p, uint8_t* smem,
                                          Shared* S, const CUtensorMap* map,
                                          int& count, int tok, int h, int b,
                                          uint64_t policy) {
  constexpr int kNB = D / 64;
  const int st = count % R::depth;
  if (!wait_bar(&S->empty[R::first + st], ((count / R::depth) & 1) ^ 1, S,
                p.status))
    return false;
  uint64_t* full = &S->full[R::first + st];
  mbar_arrive_expect_tx(full, kNB * kBox);
  for (int bx = 0; bx < kNB; ++bx)
    tma_load_4d_hint(map, smem + R::off + (st * kNB + bx) * kBox, full, bx * 64,
                     tok, h, b, policy);
  ++count;
  return true;
}
// Every load has landed before the CTA may exit.
template <class R>
__device__ __forceinline__ void ring_drain(Shared* S, int count) {
  for (int i = max(0, count - R::depth); i < count; ++i)
    drain_wait(&S->full[R::first + i % R::depth], (i / R::depth) & 1, S);
}
// The relay's part: the `count`-th tile has landed.
template <class R>
__device__ __forceinline__ bool ring_landed(const BwdParams& p, Shared* S,
                                            int count) {
  return wait_bar_warp(&S->full[R::first + count % R::depth],
                       (count / R::depth) & 1, S, p.status);
}
template <class R>
__device__ __forceinline__ void ring_hand(int count) {
  relay_arrive(kBarRing + R::first + count % R::depth);
}
// The MMA warp's part.
template <class R>
__device__ __forceinline__ void ring_take(int count) {
  relay_sync(kBarRing + R::first + count % R::depth);
}
template <class R>
__device__ __forceinline__ void ring_free(Shared* S, int count) {
  mma_commit_warp(&S->empty[R::first + count % R::depth]);
}

// After the relay's last tile: the MMA warp may still wait for arrivals that a
// failed role will not make.
__device__ __forceinline__ void relay_release(Shared* S) {
  volatile int* done = &S->mma_done;
  volatile int* abort = &S->abort;
  const uint64_t t0 = global_timer_ns();
  while (!__any_sync(~0u, *done != 0)) {
    if (__any_sync(~0u, *abort != 0)) {
      compute_arrive(kBarP);
      compute_arrive(kBarDS);
      compute_arrive(kBarDS + 1);
      for (int id = kBarRing; id < kBars; ++id) relay_arrive(id);
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

__device__ __forceinline__ void mma_finish(Shared* S) {
  mma_commit_warp(&S->drain);
  if ((threadIdx.x & 31) == 0) {
    drain_wait(&S->drain, 0, S);
    *reinterpret_cast<volatile int*>(&S->mma_done) = 1;
  }
  __syncwarp();
}

__device__ __forceinline__ uint32_t setup(Shared* S, const BwdParams& p) {
  const int warp = warp_uniform(threadIdx.x / 32);
  if (warp == kMmaWarp) {
    tmem_alloc(&S->tmem_base, kTmemCols);
    tmem_relinquish();
  }
  if (threadIdx.x == kWarpB * 32) {
    tma_prefetch_desc(&p.q_map);
    tma_prefetch_desc(&p.k_map);
    tma_prefetch_desc(&p.v_map);
    tma_prefetch_desc(&p.do_map);
  }
  if (threadIdx.x == kWarpA * 32) {
    for (int i = 0; i < kRingSlots; ++i) {
      mbar_init(&S->full[i], 1);
      mbar_init(&S->empty[i], 1);
    }
    mbar_init(&S->fixed_full, 1);
    mbar_init(&S->s_ready, 1);
    mbar_init(&S->out_full, 1);
    mbar_init(&S->drain, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&S->dp_ready[i], 1);
      mbar_init(&S->vec_full[i], 1);
      mbar_init(&S->vec_empty[i], 8);  // one arrival per compute warp
    }
    S->abort = 0;
    S->mma_done = 0;
    S->wait_limit_ns = p.wait_limit_ns ? p.wait_limit_ns : kDefaultWaitLimitNs;
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  return warp_uniform(S->tmem_base);
}

__device__ __forceinline__ void teardown(uint32_t tmem) {
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x / 32 == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// D = A B^T over the head dim, both K-major tiles at byte offsets a and b.
template <int D>
__device__ __forceinline__ void mma_nt(uint32_t sbase, uint32_t d, int a,
                                       int b) {
  constexpr uint32_t kIdesc = idesc_bf16_f32(kT, kT, 0);
  const uint32_t hi = desc_hi_sw128(1024);
  const uint32_t a_lo = desc_lo(sbase + a, 16), b_lo = desc_lo(sbase + b, 16);
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const uint32_t off = (uint32_t)((ks / 4) * kBox + (ks % 4) * 32) >> 4;
    mma_ss_warp(d, a_lo + off, b_lo + off, hi, kIdesc, ks > 0);
  }
}
// D (+)= A B, A bf16 in TMEM as the compute warps leave it (two halves of 64
// columns, each packed at the start of its own 64), B an MN-major tile.
template <int D>
__device__ __forceinline__ void mma_tn(uint32_t sbase, uint32_t d, uint32_t a,
                                       int b, bool acc) {
  constexpr uint32_t kIdesc = idesc_bf16_f32(kT, D, 1);
  const uint32_t hi = desc_hi_sw128(1024);
  const uint32_t b_lo = desc_lo(sbase + b, kBox);
#pragma unroll
  for (int kk = 0; kk < kT / 16; ++kk)
    mma_ts_warp(d, a + 64 * (kk / 4) + 8 * (kk % 4),
                b_lo + (uint32_t)(kk * 2048 >> 4), hi, kIdesc, acc || kk > 0);
}

// P = 2^(s c2 + nl) for 32 columns, in place as float32 and packed to bfloat16
// pairs; columns from `hi` on are masked where kMask.  One group of four in eight
// takes its exponentials on the FMA pipe, as in the one-shot backward.
template <bool kMask>
__device__ __forceinline__ void probs32(uint32_t (&s)[32],
                                        const float4 (&nl)[8], int c0, int hi,
                                        uint64_t c2x2, uint32_t (&pp)[16]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float4 a = nl[q];
    float x[4];
    f2_split(f2_fma(f2(__uint_as_float(s[4 * q]), __uint_as_float(s[4 * q + 1])),
                    c2x2, f2(a.x, a.y)),
             x[0], x[1]);
    f2_split(f2_fma(f2(__uint_as_float(s[4 * q + 2]),
                       __uint_as_float(s[4 * q + 3])),
                    c2x2, f2(a.z, a.w)),
             x[2], x[3]);
    if (kMask) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c0 + 4 * q + u >= hi) x[u] = -INFINITY;
    }
    if (!kMask && grad::poly_group(q)) {
      exp2_poly(x[0], x[1]);
      exp2_poly(x[2], x[3]);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = grad::ex2(x[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) s[4 * q + u] = __float_as_uint(x[u]);
    pp[2 * q] = pack_bf16(x[0], x[1]);
    pp[2 * q + 1] = pack_bf16(x[2], x[3]);
  }
}
// dS = P (dP - D) for 32 columns: P as probs32 left it, unrounded, so that dS is
// rounded once; nd holds -D.
__device__ __forceinline__ void dscores32(const uint32_t (&p)[32],
                                          const uint32_t (&dp)[32],
                                          const float4 (&nd)[8],
                                          uint32_t (&pd)[16]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float4 g = nd[q];
    float r[4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      f2_split(f2_mul(f2(__uint_as_float(p[4 * q + 2 * u]),
                         __uint_as_float(p[4 * q + 2 * u + 1])),
                      f2_add(f2(__uint_as_float(dp[4 * q + 2 * u]),
                                __uint_as_float(dp[4 * q + 2 * u + 1])),
                             u == 0 ? f2(g.x, g.y) : f2(g.z, g.w))),
               r[2 * u], r[2 * u + 1]);
    pd[2 * q] = pack_bf16(r[0], r[1]);
    pd[2 * q + 1] = pack_bf16(r[2], r[3]);
  }
}

// 32 scaled results of TMEM, where a lane has a row, as bfloat16 to rows `even` and
// `odd` of the lane and its neighbour (null: no such row).  A lane writes 32 bytes
// of both (cross_attn.cu): with the forward 295.5 us for 12288 tokens of 24 heads over
// 512 keys (298.3 without the exchange), 158.1 over 128 (160.0).
__device__ __forceinline__ void store_cols32(uint32_t taddr, float mul,
                                             bool zero, uint16_t* even,
                                             uint16_t* odd, bool wide) {
  uint32_t v[32], pk[16];
  __syncwarp();
  tmem_ld32(taddr, v);
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 16; ++i)
    pk[i] = zero ? 0u
                 : pack_bf16(__uint_as_float(v[2 * i]) * mul,
                             __uint_as_float(v[2 * i + 1]) * mul);
  const bool b = threadIdx.x & 1;
  swap_pieces(pk, b);
  if (even != nullptr) store_piece(even + 16 * b, pk, wide);
  if (odd != nullptr) store_piece(odd + 16 * b, pk + 8, wide);
}
// The two rows' places, from the first one's.
struct Rows {
  uint16_t *even, *odd;
};
__device__ __forceinline__ Rows rows_at(uint16_t* first, int64_t stride,
                                        int row, int rows) {
  return {row < rows ? first : nullptr,
          row + 1 < rows ? first + stride : nullptr};
}

// ------------------------------------------------------------------ dK, dV
// TMEM: [0,128) S^T then P^T (bf16), [128,256) dP^T then dS^T, [256,256+d) dV,
// [384,384+d) dK.  Step x: query tile x % q_tiles of head x / q_tiles of the
// group.
template <int D>
__device__ __forceinline__ void dkdv_cta(const BwdParams& p, uint8_t* smem,
                                         Shared* S, uint32_t tmem) {
  using L = DkdvLayout<D>;
  using RQ = typename L::Q;
  using RO = typename L::O;
  const int warp = warp_uniform(threadIdx.x / 32);
  const int lane = threadIdx.x % 32;
  // parts of a key tile and key tiles of a head side by side: their CTAs share
  // query tiles in L2
  int x = blockIdx.x;
  const int part = x % p.parts;
  x /= p.parts;
  const int k0 = x % p.k_tiles * kT;
  const int bh = x / p.k_tiles;
  const int hk = bh % p.kv_heads, b = bh / p.kv_heads;
  const int len = cross_keys(p.kv_len, b, p.kv_tokens);
  if (k0 >= len) {  // no key of the tile is seen; parts are not read then
    if (p.parts == 1) {
      const int rows = min(kT, p.kv_tokens - k0);
      for (int i = threadIdx.x; i < rows * (D / 8); i += kThreads) {
        const int64_t t = k0 + i / (D / 8);
        const int c = i % (D / 8) * 8;
        const uint4 z = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(p.dk + b * p.dk_str.batch +
                                  t * p.dk_str.token + hk * p.dk_str.head + c) =
            z;
        *reinterpret_cast<uint4*>(p.dv + b * p.dv_str.batch +
                                  t * p.dv_str.token + hk * p.dv_str.head + c) =
            z;
      }
    }
    return;
  }
  const int steps = p.group * p.q_tiles;
  const int x0 = (int)((int64_t)part * steps / p.parts);
  const int n = (int)((int64_t)(part + 1) * steps / p.parts) - x0;
  const int h0 = hk * p.group;

  if (warp == kWarpA) {
    if (lane == 0) {
      const uint64_t keep = l2_policy_evict_last();
      mbar_arrive_expect_tx(&S->fixed_full, 2 * L::kTile);
      for (int bx = 0; bx < L::kNB; ++bx) {
        tma_load_4d_hint(&p.k_map, smem + L::k_off + bx * kBox, &S->fixed_full,
                         bx * 64, k0, hk, b * p.k_batch, keep);
        tma_load_4d_hint(&p.v_map, smem + L::v_off + bx * kBox, &S->fixed_full,
                         bx * 64, k0, hk, b * p.v_batch, keep);
      }
      int qc = 0, oc = 0;
      for (int j = 0; j < n; ++j) {
        const int h = h0 + (int)fast_div(x0 + j, p.by_q_tiles);
        const int tok = (x0 + j - (h - h0) * p.q_tiles) * kT;
        // Test hook: waits run out, the MMA warp amid its work.
        if (p.inject_stall == 2 && j == 1 &&
            !wait_bar(&S->drain, 0, S, p.status))
          break;
        if (!ring_load<D, RO>(p, smem, S, &p.do_map, oc, tok, h,
                              b * p.do_batch, keep) ||
            !ring_load<D, RQ>(p, smem, S, &p.q_map, qc, tok, h, b * p.q_batch,
                              keep))
          break;
      }
      drain_wait(&S->fixed_full, 0, S);
      ring_drain<RO>(S, oc);
      ring_drain<RQ>(S, qc);
    }
    __syncwarp();
  } else if (warp == kRelayWarp) {
    for (int j = 0; j < n; ++j) {
      if (!ring_landed<RQ>(p, S, j)) break;
      ring_hand<RQ>(j);
      if (!ring_landed<RO>(p, S, j)) break;
      ring_hand<RO>(j);
    }
    relay_release(S);
  } else if (warp == kWarpB) {
    // 128 -log2 LSE and -D values of each step
    if (lane == 0) {
      int issued = 0;
      for (int j = 0; j < n; ++j) {
        const int h = h0 + (int)fast_div(x0 + j, p.by_q_tiles);
        const int64_t at = ((int64_t)b * p.heads + h) * p.padded +
                           (x0 + j - (h - h0) * p.q_tiles) * kT;
        const int sl = j & 1;
        if (!wait_bar(&S->vec_empty[sl], ((j >> 1) & 1) ^ 1, S, p.status))
          break;
        mbar_arrive_expect_tx(&S->vec_full[sl], 2 * kT * sizeof(float));
        bulk_load(smem + L::vec(sl, 0), p.lse2 + at, kT * sizeof(float),
                  &S->vec_full[sl]);
        bulk_load(smem + L::vec(sl, 1), p.delta + at, kT * sizeof(float),
                  &S->vec_full[sl]);
        ++issued;
      }
      for (int i = max(0, issued - 2); i < issued; ++i)
        drain_wait(&S->vec_full[i & 1], (i >> 1) & 1, S);
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    const uint32_t base = smem_addr(smem);
    auto q_at = [](int c) { return RQ::off + c % RQ::depth * L::kTile; };
    auto o_at = [](int c) { return RO::off + c % RO::depth * L::kTile; };
    // Test hook: `out_full` receives no arrival before the end.
    bool ok = (p.inject_stall != 1 ||
               wait_bar_warp(&S->out_full, 0, S, p.status)) &&
              wait_bar_warp(&S->fixed_full, 0, S, p.status);
    if (ok) {
      ring_take<RQ>(0);
      tc_fence_after();
      mma_nt<D>(base, tmem, L::k_off, q_at(0));  // S^T_0 = K Q_0^T
      mma_commit_warp(&S->s_ready);
      ring_take<RO>(0);
      tc_fence_after();
      mma_nt<D>(base, tmem + 128, L::v_off, o_at(0));  // dP^T_0 = V dO_0^T
      mma_commit_warp(&S->dp_ready[0]);
    }
    for (int j = 0; ok && j < n; ++j) {
      const uint32_t aborted = read_abort(S);
      compute_sync(kBarP);
      tc_fence_after();
      mma_tn<D>(base, tmem + 256, tmem, o_at(j), j > 0);  // dV
      ring_free<RO>(S, j);
      if (j + 1 < n) {
        ring_take<RQ>(j + 1);
        tc_fence_after();
        mma_nt<D>(base, tmem, L::k_off, q_at(j + 1));
        mma_commit_warp(&S->s_ready);
      }
      compute_sync(kBarDS);
      tc_fence_after();
      mma_tn<D>(base, tmem + 384, tmem + 128, q_at(j), j > 0);  // dK
      ring_free<RQ>(S, j);
      if (j + 1 < n) {
        ring_take<RO>(j + 1);
        tc_fence_after();
        mma_nt<D>(base, tmem + 128, L::v_off, o_at(j + 1));
        mma_commit_warp(&S->dp_ready[0]);
      }
      if (__any_sync(~0u, aborted != 0)) ok = false;
    }
    if (ok) mma_commit_warp(&S->out_full);
    mma_finish(S);
  } else {
    // Warp w owns key rows 32 (w % 4) .. + 31 (its TMEM lanes) and query columns
    // [64 hf, 64 hf + 64); its P^T and dS^T go over its own S^T and dP^T columns.
    const int hf = warp / 4;
    const int t = (warp % 4) * 32 + lane;
    const uint32_t row_t = tmem + ((uint32_t)((warp % 4) * 32) << 16);
    const uint32_t cs = 64 * hf, cp = 128 + 64 * hf;
    const uint64_t c2x2 = f2(p.scale_log2, p.scale_log2);
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      const int sl = j & 1;
      if (!(ok = wait_bar_warp(&S->vec_full[sl], (j >> 1) & 1, S, p.status)))
        break;
      const float4* nl =
          reinterpret_cast<const float4*>(smem + L::vec(sl, 0)) + 16 * hf;
      const float4* nd =
          reinterpret_cast<const float4*>(smem + L::vec(sl, 1)) + 16 * hf;
      float4 la[8], lb[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) la[q] = nl[q];
      if (!(ok = wait_bar_warp(&S->s_ready, j & 1, S, p.status))) break;
      tc_fence_after();
      uint32_t x0r[32], x1r[32], y[32], pk[16];
      tmem_ld32(row_t + cs, x0r);
      tmem_ld32(row_t + cs + 32, x1r);
#pragma unroll
      for (int q = 0; q < 8; ++q) lb[q] = nl[8 + q];
      tmem_wait_ld();
      probs32<false>(x0r, la, 0, 0, c2x2, pk);
      tmem_st16(row_t + cs, pk);
      probs32<false>(x1r, lb, 0, 0, c2x2, pk);
      tmem_st16(row_t + cs + 16, pk);
      tmem_wait_st();
      tc_fence_before();
      compute_arrive(kBarP);
#pragma unroll
      for (int q = 0; q < 8; ++q) la[q] = nd[q];
      if (!(ok = wait_bar_warp(&S->dp_ready[0], j & 1, S, p.status))) break;
      tc_fence_after();
      // half by half: there are no registers for P, dP and -D of 64 columns
      tmem_ld32(row_t + cp, y);
      tmem_wait_ld();
      dscores32(x0r, y, la, pk);
      tmem_ld32(row_t + cp + 32, y);
      tmem_st16(row_t + cp, pk);
#pragma unroll
      for (int q = 0; q < 8; ++q) la[q] = nd[8 + q];
      tmem_wait_ld();
      dscores32(x1r, y, la, pk);
      tmem_st16(row_t + cp + 16, pk);
      tmem_wait_st();
      tc_fence_before();
      compute_arrive(kBarDS);
      __syncwarp();
      if (lane == 0) mbar_arrive(&S->vec_empty[sl]);
    }
    if (ok && wait_bar_warp(&S->out_full, 0, S, p.status)) {
      tc_fence_after();
      const int row = k0 + t;
      const bool zero = row >= len;
      if (p.parts == 1) {
        const int even = row & ~1;
        const Rows dk = rows_at(p.dk + (int64_t)b * p.dk_str.batch +
                                    (int64_t)even * p.dk_str.token +
                                    (int64_t)hk * p.dk_str.head,
                                p.dk_str.token, even, p.kv_tokens);
        const Rows dv = rows_at(p.dv + (int64_t)b * p.dv_str.batch +
                                    (int64_t)even * p.dv_str.token +
                                    (int64_t)hk * p.dv_str.head,
                                p.dv_str.token, even, p.kv_tokens);
        auto at = [](uint16_t* o, int c) { return o ? o + c * 32 : o; };
#pragma unroll 1
        for (int c = hf * D / 64; c < (hf + 1) * D / 64; ++c) {
          store_cols32(row_t + 256 + c * 32, 1.f, zero, at(dv.even, c),
                       at(dv.odd, c), p.wide_v);
          store_cols32(row_t + 384 + c * 32, p.scale, zero, at(dk.even, c),
                       at(dk.odd, c), p.wide_k);
        }
      } else {
        const int64_t at = (((int64_t)part * p.batch * p.kv_heads + bh) *
                                p.k_tiles * kT + row) * D;
#pragma unroll 1
        for (int c = hf * D / 64; c < (hf + 1) * D / 64; ++c) {
          uint32_t v[32];
          __syncwarp();
          tmem_ld32(row_t + 256 + c * 32, v);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 4; ++i)
            store_32b(p.dv_part + at + c * 32 + 8 * i, v + 8 * i);
          __syncwarp();
          tmem_ld32(row_t + 384 + c * 32, v);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 4; ++i)
            store_32b(p.dk_part + at + c * 32 + 8 * i, v + 8 * i);
        }
      }
    }
  }
}

// dk and dv as the sums of their parts, in order; zeros past the last key.  A
// thread takes 8 elements of a key of both.
template <int D>
__global__ void __launch_bounds__(256)
join_kernel(const __grid_constant__ BwdParams p) {
  pdl_trigger();
  pdl_wait();
  constexpr int kPer = D / 8;
  const int64_t keys = (int64_t)p.batch * p.kv_heads * p.k_tiles * kT;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= keys * kPer) return;
  const int64_t key = i / kPer;  // of (b, hk, padded token)
  const int c = (int)(i % kPer) * 8;
  const int bh = (int)(key / (p.k_tiles * kT));
  const int t = (int)(key - (int64_t)bh * p.k_tiles * kT);
  if (t >= p.kv_tokens) return;
  const int b = bh / p.kv_heads, hk = bh % p.kv_heads;
  float sk[8] = {}, sv[8] = {};
  if (t < cross_keys(p.kv_len, b, p.kv_tokens)) {
    for (int s = 0; s < p.parts; ++s) {
      const int64_t at = (s * keys + key) * D + c;
      const float4* k4 = reinterpret_cast<const float4*>(p.dk_part + at);
      const float4* v4 = reinterpret_cast<const float4*>(p.dv_part + at);
      const float4 a = k4[0], e = k4[1], g = v4[0], h = v4[1];
      sk[0] += a.x, sk[1] += a.y, sk[2] += a.z, sk[3] += a.w;
      sk[4] += e.x, sk[5] += e.y, sk[6] += e.z, sk[7] += e.w;
      sv[0] += g.x, sv[1] += g.y, sv[2] += g.z, sv[3] += g.w;
      sv[4] += h.x, sv[5] += h.y, sv[6] += h.z, sv[7] += h.w;
    }
  }
  uint32_t ok[4], ov[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ok[e] = pack_bf16(sk[2 * e] * p.scale, sk[2 * e + 1] * p.scale);
    ov[e] = pack_bf16(sv[2 * e], sv[2 * e + 1]);
  }
  *reinterpret_cast<uint4*>(p.dk + (int64_t)b * p.dk_str.batch +
                            (int64_t)t * p.dk_str.token +
                            (int64_t)hk * p.dk_str.head + c) =
      make_uint4(ok[0], ok[1], ok[2], ok[3]);
  *reinterpret_cast<uint4*>(p.dv + (int64_t)b * p.dv_str.batch +
                            (int64_t)t * p.dv_str.token +
                            (int64_t)hk * p.dv_str.head + c) =
      make_uint4(ov[0], ov[1], ov[2], ov[3]);
}

// --------------------------------------------------------------------- dQ
// TMEM: [0,128) S, [128,256) and [384,512) dP then dS (bf16) of even and odd
// steps, [256,256+d) dQ.
__device__ __forceinline__ uint32_t dp_col(int s) { return s & 1 ? 384 : 128; }

struct Unit {
  int b, h, q0, len, n;
};
__device__ __forceinline__ void get_unit(const BwdParams& p, int x, Unit* u) {
  const uint32_t bh = fast_div(x, p.by_q_tiles);
  u->q0 = (int)(x - bh * p.q_tiles) * kT;
  u->b = (int)fast_div(bh, p.by_heads);
  u->h = (int)(bh - (uint32_t)u->b * p.heads);
  u->len = cross_keys(p.kv_len, u->b, p.kv_tokens);
  u->n = (u->len + kT - 1) / kT;
}
__device__ __forceinline__ bool next_unit(const BwdParams& p, int& x, Unit* u) {
  for (; x < p.units; x += p.dq_ctas) {
    get_unit(p, x, u);
    if (u->n > 0) {
      x += p.dq_ctas;
      return true;
    }
  }
  return false;
}

// Rows of a tile from `valid` on, zeroed by a warp (a row is 128 bytes of each
// box; the swizzle stays within rows).
template <int D>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int valid, int lane) {
  for (int bx = 0; bx < D / 64; ++bx) {
    uint4* rows = reinterpret_cast<uint4*>(tile + bx * kBox);
    for (int i = valid * 8 + lane; i < kT * 8; i += 32)
      rows[i] = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  __syncwarp();
}

template <int D>
__device__ __forceinline__ void dq_cta(const BwdParams& p, uint8_t* smem,
                                       Shared* S, uint32_t tmem, int cta) {
  using L = DqLayout<D>;
  using RQ = typename L::Q;
  using RO = typename L::O;
  using RK = typename L::K;
  using RV = typename L::V;
  const int warp = warp_uniform(threadIdx.x / 32);
  const int lane = threadIdx.x % 32;

  if (warp == kWarpA || warp == kWarpB) {
    // K_0, Q, K_1, ... and V_0, dO, V_1, ...: a unit's first K and V can be on
    // their way before the last unit's Q and dO are done with
    if (lane == 0) {
      const bool a = warp == kWarpA;
      const uint64_t once = l2_policy_evict_first(),
                     keep = l2_policy_evict_last();
      int x = cta, c = 0, r = 0;
      Unit u;
      bool ok = a || p.inject_stall != 2 ||  // test hook, as in dkdv_cta
                wait_bar(&S->drain, 0, S, p.status);
      while (ok && next_unit(p, x, &u)) {
        const int hk = (int)fast_div(u.h, p.by_group);
        for (int j = 0; ok && j < u.n; ++j) {
          ok = a ? ring_load<D, RK>(p, smem, S, &p.k_map, c, j * kT, hk,
                                    u.b * p.k_batch, keep)
                 : ring_load<D, RV>(p, smem, S, &p.v_map, c, j * kT, hk,
                                    u.b * p.v_batch, keep);
          if (ok && j == 0)
            ok = a ? ring_load<D, RQ>(p, smem, S, &p.q_map, r, u.q0, u.h,
                                      u.b * p.q_batch, once)
                   : ring_load<D, RO>(p, smem, S, &p.do_map, r, u.q0, u.h,
                                      u.b * p.do_batch, once);
        }
      }
      if (a) {
        ring_drain<RK>(S, c);
        ring_drain<RQ>(S, r);
      } else {
        ring_drain<RV>(S, c);
        ring_drain<RO>(S, r);
      }
    }
    __syncwarp();
  } else if (warp == kRelayWarp) {
    int x = cta, c = 0, r = 0;
    Unit u;
    bool ok = true;
    while (ok && next_unit(p, x, &u)) {
      for (int j = 0; ok && j < u.n; ++j, ++c) {
        // without lengths the rows past the last key lie outside the maps: zeros
        const int valid = p.kv_len != nullptr ? u.len - j * kT : kT;
        if (j == 0) {
          if (!(ok = ring_landed<RQ>(p, S, r))) break;
          ring_hand<RQ>(r);
        }
        if (!(ok = ring_landed<RK>(p, S, c))) break;
        if (valid < kT)
          zero_rows<D>(smem + RK::off + c % RK::depth * L::kTile, valid, lane);
        ring_hand<RK>(c);
        if (j == 0) {
          if (!(ok = ring_landed<RO>(p, S, r))) break;
          ring_hand<RO>(r);
        }
        if (!(ok = ring_landed<RV>(p, S, c))) break;
        if (valid < kT)
          zero_rows<D>(smem + RV::off + c % RV::depth * L::kTile, valid, lane);
        ring_hand<RV>(c);
      }
      ++r;
    }
    relay_release(S);
  } else if (warp == kMmaWarp) {
    const uint32_t base = smem_addr(smem);
    auto at = [](int off, int depth, int c) {
      return off + c % depth * L::kTile;
    };
    // Test hook: `drain` receives no arrival before the end.
    bool ok = p.inject_stall != 1 || wait_bar_warp(&S->drain, 0, S, p.status);
    int x = cta;
    Unit u, nu;
    bool have = next_unit(p, x, &u);
    bool have_next = have && next_unit(p, x, &nu);
    // S and dP of step s: tile `kc` of K and V, tile `qc` of Q and dO
    auto scores = [&](int s, int qc, bool first, bool last) {
      if (first) ring_take<RQ>(qc);
      ring_take<RK>(s);
      tc_fence_after();
      mma_nt<D>(base, tmem, at(RQ::off, RQ::depth, qc),
                at(RK::off, RK::depth, s));
      mma_commit_warp(&S->s_ready);
      if (last) ring_free<RQ>(S, qc);
      if (first) ring_take<RO>(qc);
      ring_take<RV>(s);
      tc_fence_after();
      mma_nt<D>(base, tmem + dp_col(s), at(RO::off, RO::depth, qc),
                at(RV::off, RV::depth, s));
      mma_commit_warp(&S->dp_ready[s & 1]);
      ring_free<RV>(S, s);
      if (last) ring_free<RO>(S, qc);
    };
    int s = 0, j = 0, qc = 0;
    if (ok && have) scores(0, 0, true, u.n == 1);
    while (ok && have) {
      const uint32_t aborted = read_abort(S);
      const bool last = j == u.n - 1;
      compute_sync(kBarP);
      if (!last)
        scores(s + 1, qc, false, j + 1 == u.n - 1);
      else if (have_next)
        scores(s + 1, qc + 1, true, nu.n == 1);
      compute_sync(kBarDS + (s & 1));
      tc_fence_after();
      mma_tn<D>(base, tmem + 256, tmem + dp_col(s),
                at(RK::off, RK::depth, s), j > 0);
      ring_free<RK>(S, s);
      if (last) mma_commit_warp(&S->out_full);
      ++s;
      ++j;
      if (last) {
        j = 0;
        ++qc;
        u = nu;
        have = have_next;
        have_next = have && next_unit(p, x, &nu);
      }
      if (__any_sync(~0u, aborted != 0)) ok = false;
    }
    mma_finish(S);
  } else {
    // Warp w owns query rows 32 (w % 4) .. + 31 and key columns [64 hf, + 64).
    const int hf = warp / 4;
    const int t = (warp % 4) * 32 + lane;
    const uint32_t row_t = tmem + ((uint32_t)((warp % 4) * 32) << 16);
    const uint64_t c2x2 = f2(p.scale_log2, p.scale_log2);
    int owed = -1;  // the unit whose dQ is still to be written
    bool ok = true;
    int s = 0, done = 0;
    auto write_out = [&]() {
      if (!(ok = wait_bar_warp(&S->out_full, done & 1, S, p.status))) return;
      ++done;
      tc_fence_after();
      Unit u;
      get_unit(p, owed, &u);
      const int even = u.q0 + (t & ~1);
      const Rows o = rows_at(p.dq + (int64_t)u.b * p.dq_str.batch +
                                 (int64_t)even * p.dq_str.token +
                                 (int64_t)u.h * p.dq_str.head,
                             p.dq_str.token, even, p.q_tokens);
#pragma unroll 1
      for (int c = hf * D / 64; c < (hf + 1) * D / 64; ++c)
        store_cols32(row_t + 256 + c * 32, p.scale, false,
                     o.even ? o.even + c * 32 : nullptr,
                     o.odd ? o.odd + c * 32 : nullptr, p.wide_q);
      tc_fence_before();
    };
    // A unit's row values lie at kT times its number; the next one's are asked
    // for a unit ahead.
    float nl_next = p.lse2[(int64_t)cta * kT + t];
    float nd_next = p.delta[(int64_t)cta * kT + t];
    for (int x = cta; ok && x < p.units; x += p.dq_ctas) {
      Unit u;
      get_unit(p, x, &u);
      const float nl_row = nl_next, nd_row = nd_next;
      if (x + p.dq_ctas < p.units) {
        nl_next = p.lse2[(int64_t)(x + p.dq_ctas) * kT + t];
        nd_next = p.delta[(int64_t)(x + p.dq_ctas) * kT + t];
      }
      if (u.n == 0) {  // sees no key
        const int row = u.q0 + t;
        uint16_t* dst = p.dq + (int64_t)u.b * p.dq_str.batch +
                        (int64_t)row * p.dq_str.token +
                        (int64_t)u.h * p.dq_str.head;
        if (row < p.q_tokens)
          for (int c = hf * D / 2; c < (hf + 1) * D / 2; c += 8)
            *reinterpret_cast<uint4*>(dst + c) = make_uint4(0, 0, 0, 0);
        __syncwarp();
        continue;
      }
      float4 nl_v[8], nd_v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        nl_v[q] = make_float4(nl_row, nl_row, nl_row, nl_row);
        nd_v[q] = make_float4(nd_row, nd_row, nd_row, nd_row);
      }
      for (int j = 0; j < u.n; ++j, ++s) {
        if (!(ok = wait_bar_warp(&S->s_ready, s & 1, S, p.status))) break;
        tc_fence_after();
        const int hi = u.len - j * kT - 64 * hf;  // visible columns
        uint32_t x0[32], x1[32], y0[32], y1[32], pk[16];
        tmem_ld32(row_t + 64 * hf, x0);
        tmem_ld32(row_t + 64 * hf + 32, x1);
        tmem_wait_ld();
        if (hi < 64) {
          probs32<true>(x0, nl_v, 0, hi, c2x2, pk);
          probs32<true>(x1, nl_v, 32, hi, c2x2, pk);
        } else {
          probs32<false>(x0, nl_v, 0, hi, c2x2, pk);
          probs32<false>(x1, nl_v, 32, hi, c2x2, pk);
        }
        tc_fence_before();
        compute_arrive(kBarP);
        if (j == 0 && owed >= 0) {
          write_out();
          if (!ok) break;
        }
        if (!(ok = wait_bar_warp(&S->dp_ready[s & 1], (s >> 1) & 1, S,
                                 p.status)))
          break;
        tc_fence_after();
        const uint32_t cp = dp_col(s) + 64 * hf;
        tmem_ld32(row_t + cp, y0);
        tmem_ld32(row_t + cp + 32, y1);
        tmem_wait_ld();
        dscores32(x0, y0, nd_v, pk);
        tmem_st16(row_t + cp, pk);
        dscores32(x1, y1, nd_v, pk);
        tmem_st16(row_t + cp + 16, pk);
        tmem_wait_st();
        tc_fence_before();
        compute_arrive(kBarDS + (s & 1));
      }
      owed = x;
    }
    if (ok && owed >= 0) write_out();
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
grads_kernel(const __grid_constant__ BwdParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  // The layouts leave no room to round the base up.
  if ((smem_addr(smem) & 1023u) != 0) {
    if (threadIdx.x == 0 && p.status != nullptr)
      atomicExch(p.status, kDevBounds);
    return;
  }
  Shared* S = reinterpret_cast<Shared*>(smem);
  const uint32_t tmem = setup(S, p);
  pdl_trigger();
  pdl_wait();
  if ((int)blockIdx.x < p.dkdv_ctas)
    dkdv_cta<D>(p, smem, S, tmem);
  else
    dq_cta<D>(p, smem, S, tmem, (int)blockIdx.x - p.dkdv_ctas);
  teardown(tmem);
}

// -D_i = -<dO_i, O_i> and minus the log-sum-exp in log2 units (negated: both
// enter packed multiply-adds as addends), zeros past the last token.  d / 8
// lanes to a row, all loads of a block before its first product.
constexpr int kRowTokens = 64;
template <int D>
__global__ void __launch_bounds__(256)
rows_kernel(const __grid_constant__ CrossBwdArgs a, float* lse2, float* delta,
            int padded, FastDiv by_tiles, FastDiv by_heads) {
  constexpr int kLanes = D / 8, kPer = 256 / kLanes;
  constexpr int kPasses = kRowTokens / kPer;
  __shared__ float red[kRowTokens];
  pdl_trigger();
  pdl_wait();
  const CrossArgs& f = a.f;
  const int bh = (int)fast_div(blockIdx.x, by_tiles);
  const int t0 = ((int)blockIdx.x - bh * (padded / kRowTokens)) * kRowTokens;
  const int b = (int)fast_div(bh, by_heads), h = bh - b * f.heads;
  const int sub = threadIdx.x / kLanes, piece = threadIdx.x % kLanes;
  const uint16_t* o = f.o + (int64_t)b * f.o_str.batch +
                      (int64_t)h * f.o_str.head + piece * 8;
  const uint16_t* g = a.dout + (int64_t)b * a.dout_str.batch +
                      (int64_t)h * a.dout_str.head + piece * 8;
  uint4 x[kPasses], y[kPasses];
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int64_t tok = t0 + u * kPer + sub;
    x[u] = y[u] = make_uint4(0, 0, 0, 0);
    if (tok < f.q_tokens) {
      x[u] = __ldcs(reinterpret_cast<const uint4*>(o + tok * f.o_str.token));
      y[u] = __ldg(reinterpret_cast<const uint4*>(g + tok * a.dout_str.token));
    }
  }
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
    const uint32_t ys[4] = {y[u].x, y[u].y, y[u].z, y[u].w};
    float acc = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc = fmaf(bf16_lo(xs[e]), bf16_lo(ys[e]), acc);
      acc = fmaf(bf16_hi(xs[e]), bf16_hi(ys[e]), acc);
    }
#pragma unroll
    for (int m = kLanes / 2; m > 0; m >>= 1)
      acc += __shfl_xor_sync(~0u, acc, m);
    if (piece == 0) red[u * kPer + sub] = acc;
  }
  __syncthreads();
  if (threadIdx.x < kRowTokens) {
    const int tok = t0 + threadIdx.x;
    const bool in = tok < f.q_tokens;
    const int64_t i = (int64_t)bh * padded + tok;
    delta[i] = in ? -red[threadIdx.x] : 0.f;
    lse2[i] = in ? -f.lse[(int64_t)bh * f.q_tokens + tok] * 1.4426950408889634f
                 : 0.f;
  }
}

// ------------------------------------------------------------------ host

int64_t pad_rows(int64_t n) { return (n + kT - 1) / kT * kT; }

// CTAs of the parts do not depend on the device at hand: the scratch size is
// asked for on the host, possibly without one.
constexpr int kSms = 152;

// Ranges of a key tile's `steps` query tiles, four at most: the number that ends
// first, a CTA taking about two steps' time to start and to end and a part's
// results about a quarter of one to join.  Three for 96 tiles of 96 steps (229 us
// with dq, 238 without ranges, 259 with six), three for 48 of 52 (60, 83 and 67),
// four for 16 of 52 (40, 69 and 39).
int key_parts(int64_t tiles, int64_t steps) {
  int best = 1;
  double least = 1e300;
  for (int s = 1; s <= 4 && s <= steps; ++s) {
    const double waves = (double)((tiles * s + kSms - 1) / kSms);
    const double cost =
        waves * ((double)((steps + s - 1) / s) + 2.0) +
        (s > 1 ? 2.0 + 0.25 * (double)(tiles * s) / kSms : 0.0);
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}
// CTAs of dq to an SM: few enough units in each to fill the end of a launch, with
// one 3 to 5 % more, with three no less.
constexpr int kDqWaves = 2;

// Parts are written in pieces of 32 bytes; the caller's scratch lies on 16.
constexpr uintptr_t kPartAlign = 32;

struct ScratchLayout {
  int64_t rows, part;  // floats of one row vector, of dk's (dv's) parts
  int parts;
};
ScratchLayout layout(int64_t batch, int64_t heads, int64_t kv_heads, int64_t d,
                     int64_t q_tokens, int64_t kv_tokens) {
  ScratchLayout l;
  l.rows = batch * heads * pad_rows(q_tokens);
  const int64_t k_tiles = pad_rows(kv_tokens) / kT;
  const int64_t q_tiles = pad_rows(q_tokens) / kT;
  const int64_t tiles = batch * kv_heads * k_tiles;
  l.parts = key_parts(tiles, heads / kv_heads * q_tiles);
  l.part = l.parts > 1 ? l.parts * tiles * kT * d : 0;
  return l;
}

bool wide_rows(const void* p, const Strides& s) {
  return ((uintptr_t)p & 31) == 0 && s.batch % 16 == 0 && s.token % 16 == 0 &&
         s.head % 16 == 0;
}

template <int D>
cudaError_t launch_d(const CrossBwdArgs& a, cudaStream_t stream) {
  const CrossArgs& f = a.f;
  BwdParams p;
  memset(&p, 0, sizeof(p));
  if (!cross_map(&p.q_map, f.q, D, f.q_tokens, f.heads, f.batch, f.q_str,
                 &p.q_batch) ||
      !cross_map(&p.do_map, a.dout, D, f.q_tokens, f.heads, f.batch,
                 a.dout_str, &p.do_batch) ||
      !cross_map(&p.k_map, f.k, D, f.kv_tokens, f.kv_heads, f.batch, f.k_str,
                 &p.k_batch) ||
      !cross_map(&p.v_map, f.v, D, f.kv_tokens, f.kv_heads, f.batch, f.v_str,
                 &p.v_batch))
    return cudaErrorInvalidValue;
  const ScratchLayout l =
      layout(f.batch, f.heads, f.kv_heads, D, f.q_tokens, f.kv_tokens);
  float* lse2 = a.scratch;
  float* delta = lse2 + l.rows;
  p.lse2 = lse2;
  p.delta = delta;
  p.dk_part = reinterpret_cast<float*>(
      ((uintptr_t)(delta + l.rows) + kPartAlign - 1) & ~(kPartAlign - 1));
  p.dv_part = p.dk_part + l.part;
  p.parts = l.parts;
  p.dq = a.dq;
  p.dk = a.dk;
  p.dv = a.dv;
  p.dq_str = a.dq_str;
  p.dk_str = a.dk_str;
  p.dv_str = a.dv_str;
  p.kv_len = f.kv_len;
  p.batch = f.batch;
  p.heads = f.heads;
  p.kv_heads = f.kv_heads;
  p.group = f.heads / f.kv_heads;
  p.q_tokens = f.q_tokens;
  p.kv_tokens = f.kv_tokens;
  p.padded = (int32_t)pad_rows(f.q_tokens);
  p.q_tiles = p.padded / kT;
  p.k_tiles = (int32_t)(pad_rows(f.kv_tokens) / kT);
  p.units = p.q_tiles * f.heads * f.batch;
  p.by_q_tiles = make_div((uint32_t)p.q_tiles);
  p.by_heads = make_div((uint32_t)f.heads);
  p.by_group = make_div((uint32_t)p.group);
  p.wide_q = wide_rows(a.dq, a.dq_str);
  p.wide_k = wide_rows(a.dk, a.dk_str);
  p.wide_v = wide_rows(a.dv, a.dv_str);
  p.scale = f.scale;
  p.scale_log2 = f.scale * 1.4426950408889634f;
  p.status = f.status;
  p.inject_stall = f.inject_stall;
  p.wait_limit_ns = f.wait_limit_ns;

  static_assert(DqLayout<D>::bytes <= 227 * 1024 &&
                    DkdvLayout<D>::bytes <= 227 * 1024,
                "shared memory");
  const int row_tiles = p.padded / kRowTokens;
  cudaError_t e = launch_pdl(
      rows_kernel<D>, dim3((unsigned)(f.batch * f.heads * row_tiles)),
      dim3(256), 0, stream, a, lse2, delta, p.padded,
      make_div((uint32_t)row_tiles), p.by_heads);
  constexpr int smem = std::max(DkdvLayout<D>::bytes, DqLayout<D>::bytes);
  if (e == cudaSuccess)
    e = allow_smem<grads_kernel<D>>(smem, f.device);
  if (e != cudaSuccess) return e;
  const int tiles = f.batch * f.kv_heads * p.k_tiles;
  p.dkdv_ctas = tiles * p.parts;
  p.dq_ctas = std::min(p.units, kDqWaves * f.sms);
  e = launch_pdl(grads_kernel<D>, dim3((unsigned)(p.dkdv_ctas + p.dq_ctas)),
                 dim3(kThreads), smem, stream, p);
  if (e != cudaSuccess || p.parts == 1) return e;
  return launch_pdl(join_kernel<D>,
                    dim3((unsigned)((int64_t)tiles * kT * (D / 8) / 256)),
                    dim3(256), 0, stream, p);
}

}  // namespace

size_t cross_bwd_scratch_floats(int32_t batch, int32_t heads, int32_t kv_heads,
                                int32_t head_dim, int32_t q_tokens,
                                int32_t kv_tokens) {
  const ScratchLayout l =
      layout(batch, heads, kv_heads, head_dim, q_tokens, kv_tokens);
  const int64_t pad = l.part > 0 ? (kPartAlign - 16) / sizeof(float) : 0;
  return (size_t)(2 * l.rows + 2 * l.part + pad);
}

cudaError_t launch_cross_attn_bwd(const CrossBwdArgs& a, cudaStream_t stream) {
  return a.f.head_dim == 64 ? launch_d<64>(a, stream)
                            : launch_d<128>(a, stream);
}

}  // namespace fastvr
