// Gated feed-forward, h = act(x Wg^T) o (x Wu^T), and its gradients, on
// tcgen05 tensor cores with CTA pairs.
//
// With dg = dh o u o act'(g) and du = dh o act(g) (slope_kernel), every product
// is a sum over an axis that either operand has as its rows or its columns:
//   forward  g, u [tokens, hidden]  = x W^T        x and W by rows
//   dx       [tokens, dim] = dg Wg + du Wu         dg by rows, W by columns
//   dW       [hidden, dim] = dg^T x, du^T x        dg and x by columns
// so one kernel serves all: TMA brings 128-byte-swizzled boxes of 64 columns,
// which the MMA's descriptors read as K-major (rows) or MN-major (columns)
// operands, and nothing is transposed in memory.  A copy brings 16 KB where it
// can: with two copies of 8 KB for one operand the 1080p chunk took 242 us
// instead of 228.
//
// A pair of CTAs owns a 256 x 256 tile of results (a forward tile: 128 columns
// of g and the same 128 of u, whose product is formed in the epilogue, so g and
// u need not leave the SM).  Each CTA loads 128 rows of A and 128 of B's 256,
// 32 KB for 64 steps of the sum: half of what a CTA alone would load for the
// same products, which L2 could not deliver.  Persistent: warps 0 and 2 load A and B
// (six stages), warp 1 of the even CTA issues the MMAs of both, warps 4-11 form and
// store the results from one half of TMEM while the next tile accumulates in
// the other.  Where there are too few tiles for all pairs they are half as wide.
// Measured: 16320 x 1536 to 4096 in 227 to 241 us one after another (1700 to 1810
// TFLOP/s at the power cap, a median of 1500 MHz; its bytes take 31), 203 to 213 alone
// after a pause (1830 MHz), 92 % of the tensor pipe's cycles either way; 12288 tokens
// with g and u kept in 175 (83 %), dx and both dW of these in 335 to 353 (89 %; 1750
// TFLOP/s and more).  Every wait is bounded, as in chunk_attn_fwd.cu.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "fastvr_internal.h"
#include "ffn_act.cuh"
#include "ffn_tiles.h"
#include "sm100_ptx.cuh"

namespace fastvr {
namespace {

using namespace ffn;
using namespace sm100;

constexpr int kThreads = 384;
constexpr int kStages = 6;
constexpr int kOperand = kHalf * kStep * 2;  // bytes of one operand's stage
constexpr uint32_t kTmemCols = 512;     // two tiles' results
constexpr uint64_t kDefaultWaitLimitNs = 4000000000ull;
constexpr uint64_t kAbortGraceNs = 1000000;

struct PairParams {
  // x; gate and up weights; dg and du, by rows (dx) and by columns (dW)
  CUtensorMap x, w[2], d[2], dt[2];
  // results: forward h, g, u; backward dx, dWg, dWu
  CUtensorMap out[3];
  Division div;             // which tiles a pair takes (ffn_tiles.h)
  int32_t half_steps;       // dx: steps of dg Wg
  int32_t save;             // forward: g and u are wanted
  // by columns, a copy takes all the columns that a CTA needs: dim, hidden are
  // whole boxes
  int32_t dim_boxes, hidden_boxes;
  int* status;
  int32_t inject_stall;
  uint64_t wait_limit_ns;
};

struct Shared {
  uint64_t full[kStages], empty[kStages];
  uint64_t acc_full[2], acc_empty[2], drain;
  uint32_t tmem_base;
  int abort;
  uint64_t wait_limit_ns;
};
// Results on their way out: a box of 128 rows by 64 columns for each half of the
// storing warps.
constexpr int kBoxBytes = kHalf * 128;
constexpr int kStaging = kStages * 2 * kOperand;
constexpr int kSharedBytes = kStaging + 2 * kBoxBytes;
constexpr int kSmem = kSharedBytes + (int)sizeof(Shared) + 1024;

__device__ __forceinline__ bool give_up(Shared* S, uint64_t t0, int* status) {
  if (*reinterpret_cast<volatile int*>(&S->abort)) return true;
  if (global_timer_ns() - t0 <= S->wait_limit_ns) return false;
  *reinterpret_cast<volatile int*>(&S->abort) = 1;
  if (status != nullptr) atomicExch(status, kDevTimeout);
  return true;
}
// Bounded waits: one thread's, and a whole warp's that stays converged.  The
// barriers are arrived at from both CTAs of the pair.
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity,
                                         Shared* S, int* status) {
  if (mbar_try_wait_cluster(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait_cluster(bar, parity))
    if (give_up(S, t0, status)) return false;
  return true;
}
__device__ __forceinline__ bool wait_bar_warp(uint64_t* bar, uint32_t parity,
                                              Shared* S, int* status) {
  if (__all_sync(~0u, mbar_try_wait_cluster(bar, parity))) return true;
  const uint64_t t0 = global_timer_ns();
  while (!__all_sync(~0u, mbar_try_wait_cluster(bar, parity)))
    if (__any_sync(~0u, give_up(S, t0, status))) return false;
  return true;
}
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity,
                                           const Shared* S) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait_cluster(bar, parity))
    if (global_timer_ns() - t0 > S->wait_limit_ns) return;
}

// An operand by columns: `boxes` of 64 columns from col on, 64 rows from row on.
__device__ __forceinline__ void load_columns(const CUtensorMap* map,
                                             uint8_t* dst, uint32_t bar,
                                             int col, int row, int boxes,
                                             bool whole) {
  if (whole) {
    tma_load_3d_pair(map, dst, bar, 0, row, col / 64);
  } else {
    for (int x = 0; x < boxes; ++x)
      tma_load_3d_pair(map, dst + x * (kOperand / 2), bar, col + 64 * x, row,
                       0);
  }
}

// 32 results of row r, from column c of its box on, as bfloat16 into the box
// (128-byte rows, 16-byte piece k at k ^ (r % 8)).
__device__ __forceinline__ void stage_row32(uint8_t* box, int r, int c,
                                            const uint32_t (&pk)[16]) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<uint4*>(box + r * 128 + (((c / 8 + q) ^ (r & 7)) << 4)) =
        make_uint4(pk[4 * q], pk[4 * q + 1], pk[4 * q + 2], pk[4 * q + 3]);
}
// The four warps that share a box (named barrier 1 + half).
__device__ __forceinline__ void box_sync(int hf) {
  asm volatile("bar.sync %0, 128;" ::"r"(1 + hf) : "memory");
}
// The box may be written again / goes out to (col, row) of a map.  The first
// answers whether the four warps' waits have all ended well: where a wait ran out
// for some of them, none goes on, or those would wait for the others here.
__device__ __forceinline__ bool box_begin(int hf, bool leader, bool ok) {
  if (leader) bulk_wait_read0();
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, %2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"((uint32_t)ok), "r"(1 + hf)
      : "memory");
  return all != 0;
}
__device__ __forceinline__ void box_end(const CUtensorMap* map, uint8_t* box,
                                        int hf, bool leader, int col, int row,
                                        const Tiles& shape) {
  fence_proxy_async_smem();
  box_sync(hf);
  if (leader && col < shape.cols && row < shape.rows) {
    tma_store_2d(map, box, col, row);
    bulk_commit_group();
  }
}

__device__ __forceinline__ void pack_row32(const uint32_t (&v)[32],
                                           uint32_t (&pk)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    pk[i] = bf16_pack(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
}

// kAct: the forward's activation; -1: backward.
template <int kAct>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
pair_kernel(const __grid_constant__ PairParams p) {
  constexpr bool kBackward = kAct < 0;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Shared* S = reinterpret_cast<Shared*>(smem + kSharedBytes);
  const int warp = warp_uniform(threadIdx.x / 32);
  const int lane = threadIdx.x % 32;
  const int rank = (int)cluster_rank();
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

  if (warp == 1) tmem_alloc_pair(&S->tmem_base, kTmemCols);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&S->full[s], 1);
      mbar_init(&S->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&S->acc_full[b], 1);
      mbar_init(&S->acc_empty[b], 16);  // the storing warps of both CTAs
    }
    mbar_init(&S->drain, 1);
    S->abort = 0;
    S->wait_limit_ns = p.wait_limit_ns ? p.wait_limit_ns : kDefaultWaitLimitNs;
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = S->tmem_base;
  pdl_trigger();
  pdl_wait();
  Work w;

  if (warp == 0 || warp == 2) {
    // A's and B's tiles: one thread for both would need longer than a step's
    // products (229 us against 259 for the 1080p chunk with three copies a step)
    const bool first = warp == 0;
    if (lane == 0) {
      int it = 0;
      bool ok = true;
      for (int i = 0; ok && nth_tile(p.div, pair, pairs, i, &w); ++i) {
        const int b_boxes = 2 - w.narrow;
        for (int s = 0; s < w.steps; ++s, ++it) {
          const int st = it % kStages;
          if (!(ok = wait_bar(&S->empty[st], ((it / kStages) & 1) ^ 1, S,
                              p.status)))
            break;
          uint8_t* a = smem + st * 2 * kOperand;
          uint8_t* b = a + kOperand;
          // both CTAs' bytes count on the even CTA's barrier
          const uint32_t bar = cluster_addr(&S->full[st], 0);
          if (first && rank == 0)
            mbar_arrive_expect_tx(&S->full[st], (2 + b_boxes) * kOperand);
          if (!kBackward) {
            if (first)
              tma_load_2d_pair(&p.x, a, bar, s * kStep, w.m0 + rank * kHalf);
            else
              tma_load_2d_pair(&p.w[rank], b, bar, s * kStep, w.n0);
          } else if (w.kind == kDx) {
            const int up = s >= p.half_steps;
            const int k = (s - up * p.half_steps) * kStep;
            if (first)
              tma_load_2d_pair(&p.d[up], a, bar, k, w.m0 + rank * kHalf);
            else
              load_columns(&p.w[up], b, bar, w.n0 + rank * b_boxes * 64, k,
                           b_boxes, p.dim_boxes);
          } else if (first) {
            load_columns(&p.dt[w.which], a, bar, w.m0 + rank * kHalf,
                         s * kStep, 2, p.hidden_boxes);
          } else {
            load_columns(&p.x, b, bar, w.n0 + rank * b_boxes * 64, s * kStep,
                         b_boxes, p.dim_boxes);
          }
        }
      }
      // every load has landed before the pair exits
      if (first && rank == 0)
        for (int i = max(0, it - kStages); i < it; ++i)
          drain_wait(&S->full[i % kStages], (i / kStages) & 1, S);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t base = smem_addr(smem);
      // Test hook: `drain` receives no arrival before the end, so this wait
      // runs out and exercises the abort path.
      bool ok = !p.inject_stall || wait_bar_warp(&S->drain, 0, S, p.status);
      int it = 0;
      Work next;
      bool have = nth_tile(p.div, pair, pairs, 0, &next);
      for (int i = 0; ok && have; ++i) {
        w = next;
        const int buf = i & 1;
        if (!(ok = wait_bar_warp(&S->acc_empty[buf], ((i >> 1) & 1) ^ 1, S,
                                 p.status)))
          break;
        tc_fence_after();
        // K-major: 16 elements are 32 bytes of a row, 8 rows 1024 bytes apart.
        // MN-major: 16 elements are 16 rows of 128 bytes, 64 of the other axis
        // a box of 64 rows.
        const bool a_mn = kBackward && w.kind == kDw, b_mn = kBackward;
        const uint32_t idesc =
            idesc_bf16_f32(256, w.narrow ? 128 : 256, b_mn, a_mn);
        const uint32_t hi = desc_hi_sw128(1024);
        const uint32_t a_lbo = a_mn ? kOperand / 2 : 16;
        const uint32_t b_lbo = b_mn ? kOperand / 2 : 16;
        const uint32_t a_step = (a_mn ? 2048 : 32) >> 4;
        const uint32_t b_step = (b_mn ? 2048 : 32) >> 4;
        for (int s = 0; s < w.steps; ++s, ++it) {
          const int st = it % kStages;
          if (!(ok = wait_bar_warp(&S->full[st], (it / kStages) & 1, S,
                                   p.status)))
            break;
          tc_fence_after();
          const uint32_t a_lo = desc_lo(base + st * 2 * kOperand, a_lbo);
          const uint32_t b_lo =
              desc_lo(base + st * 2 * kOperand + kOperand, b_lbo);
#pragma unroll
          for (int k = 0; k < kStep / 16; ++k)
            mma_ss_pair_warp(tmem + buf * 256, a_lo + k * a_step, hi,
                             b_lo + k * b_step, hi, idesc, (s | k) != 0);
          mma_commit_pair_warp(&S->empty[st]);
          // found while the first step's products run
          if (s == 0) have = nth_tile(p.div, pair, pairs, i + 1, &next);
        }
        if (ok) mma_commit_pair_warp(&S->acc_full[buf]);
      }
      mma_commit_pair_warp(&S->drain);
      if (lane == 0) drain_wait(&S->drain, 0, S);
      __syncwarp();
    }
  } else if (warp >= 4) {
    const int quarter = warp % 4, hf = (warp - 4) / 4;
    const int r = quarter * 32 + lane;
    const bool leader = r == 0;
    uint8_t* box = smem + kStaging + hf * kBoxBytes;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    bool ok = true;
    for (int i = 0; ok && nth_tile(p.div, pair, pairs, i, &w); ++i) {
      const int buf = i & 1;
      ok = wait_bar_warp(&S->acc_full[buf], (i >> 1) & 1, S, p.status);
      tc_fence_after();
      const Tiles& shape = p.div.tile[kBackward && w.kind != p.div.kind[0]];
      const int row = w.m0 + rank * kHalf;
      const uint32_t acc = tmem + buf * 256 + lanes;
      const uint32_t freed = cluster_addr(&S->acc_empty[buf], 0);
      uint32_t pk[16];
      if (!kBackward && w.narrow && hf == 1) {
        // one box of columns: the other half's
        if (!ok) break;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(freed);
      } else if (!kBackward) {
        // h, then g and u where they are kept: in bfloat16, since in float32 they
        // would double the 201 MB that a clip's forward writes for them.  With dg
        // and du the gradients are off by 3.0e-3 in the 2-norm (rounding the results
        // alone by 1.7e-3).
        const int rounds = p.save ? 3 : 1;
        const int col = w.n0 + hf * 64;
        const int u_col = w.narrow ? 64 : 128;
        for (int x = 0; x < rounds; ++x) {
          if (!(ok = box_begin(hf, leader, ok))) break;
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
            uint32_t g[32], u[32];
            if (x != 2) tmem_ld32(acc + hf * 64 + c, g);
            if (x != 1) tmem_ld32(acc + u_col + hf * 64 + c, u);
            tmem_wait_ld();
            if (x == 0) {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                pk[e] = bf16_pack(activation<kAct>(__uint_as_float(g[2 * e])) *
                                      __uint_as_float(u[2 * e]),
                                  activation<kAct>(__uint_as_float(g[2 * e + 1])) *
                                      __uint_as_float(u[2 * e + 1]));
              }
            } else if (x == 1) {
              pack_row32(g, pk);
            } else {
              pack_row32(u, pk);
            }
            stage_row32(box, r, c, pk);
          }
          if (x == rounds - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(freed);
          }
          box_end(&p.out[x], box, hf, leader, col, row, shape);
        }
      } else {
        const CUtensorMap* map = &p.out[w.kind == kDx ? 0 : 1 + w.which];
        const int boxes = 2 - w.narrow;
        for (int x = 0; x < boxes; ++x) {
          const int col = (hf * boxes + x) * 64;
          if (!(ok = box_begin(hf, leader, ok))) break;
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
            uint32_t v[32];
            tmem_ld32(acc + col + c, v);
            tmem_wait_ld();
            pack_row32(v, pk);
            stage_row32(box, r, c, pk);
          }
          if (x == boxes - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(freed);
          }
          box_end(map, box, hf, leader, w.n0 + col, row, shape);
        }
      }
    }
    if (leader) bulk_wait_group0();
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  // The odd CTA's barriers have had their last arrivals once its `drain` has;
  // after a failed wait its last loads get the time to land.
  if (warp == 1 && lane == 0) {
    if (rank == 1) drain_wait(&S->drain, 0, S);
    if (S->abort) {
      const uint64_t t0 = global_timer_ns();
      while (global_timer_ns() - t0 < kAbortGraceNs) {
      }
    }
  }
  __syncwarp();
  cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

// dg = dh o u o act'(g), du = dh o act(g): memory-bound, five bfloat16 tensors
// once each, 16 bytes of each to a thread (12288 x 4096: 71 us, 7.1 TB/s with what
// L2 still holds).  Float32 inside; dg and du are
// rounded to bfloat16 because the tensor cores take them so.
template <int kAct>
__global__ void __launch_bounds__(256) slope_kernel(FfnBwdArgs a) {
  pdl_trigger();
  pdl_wait();
  const int64_t n = (int64_t)a.f.tokens * a.f.hidden / 8;
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const uint4 g = reinterpret_cast<const uint4*>(a.f.g)[i];
    const uint4 u = reinterpret_cast<const uint4*>(a.f.u)[i];
    const uint4 d = reinterpret_cast<const uint4*>(a.dh)[i];
    const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, uw[4] = {u.x, u.y, u.z, u.w},
                   dw[4] = {d.x, d.y, d.z, d.w};
    uint32_t og[4], ou[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float s0, s1;
      const float a0 = activation<kAct>(bf16_lo(gw[e]), &s0);
      const float a1 = activation<kAct>(bf16_hi(gw[e]), &s1);
      og[e] = bf16_pack(bf16_lo(dw[e]) * bf16_lo(uw[e]) * s0,
                        bf16_hi(dw[e]) * bf16_hi(uw[e]) * s1);
      ou[e] = bf16_pack(bf16_lo(dw[e]) * a0, bf16_hi(dw[e]) * a1);
    }
    reinterpret_cast<uint4*>(a.dg)[i] = make_uint4(og[0], og[1], og[2], og[3]);
    reinterpret_cast<uint4*>(a.du)[i] = make_uint4(ou[0], ou[1], ou[2], ou[3]);
  }
}

// ------------------------------------------------------------------ host

// [rows, cols] bfloat16, boxes of 64 columns by `box_rows` rows.
bool make_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols,
              int64_t row_elems, int box_rows) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (enc == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)row_elems * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base),
             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same by columns, boxes of 64 rows: where the columns are whole boxes they
// become an axis of boxes, `boxes` of which a copy takes.
bool make_column_map(CUtensorMap* m, const void* base, int64_t rows,
                     int64_t cols, int64_t row_elems, int boxes) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (enc == nullptr) return false;
  const bool whole = cols % 64 == 0;
  const cuuint64_t dims[3] = {(cuuint64_t)(whole ? 64 : cols), (cuuint64_t)rows,
                              (cuuint64_t)(whole ? cols / 64 : 1)};
  const cuuint64_t strides[2] = {(cuuint64_t)row_elems * 2, 128};
  const cuuint32_t box[3] = {64, kStep, (cuuint32_t)(whole ? boxes : 1)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base),
             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kAct>
cudaError_t launch_pairs(PairParams& p, int pairs, const FfnArgs& a,
                         cudaStream_t stream) {
  p.status = a.status;
  p.inject_stall = a.inject_stall;
  p.wait_limit_ns = a.wait_limit_ns;
  const cudaError_t e = allow_smem<pair_kernel<kAct>>(kSmem, a.device);
  if (e != cudaSuccess) return e;
  return launch_pdl(pair_kernel<kAct>, dim3(2 * pairs), dim3(kThreads),
                    kSmem, stream, p);
}

}  // namespace

cudaError_t launch_ffn_fwd(const FfnArgs& a, cudaStream_t stream) {
  if (ffn_few_rows(a.tokens)) return launch_ffn_rows(a, stream);
  PairParams p;
  memset(&p, 0, sizeof(p));
  int pairs;
  p.div = divide_fwd(a.tokens, a.dim, a.hidden, a.sms, &pairs);
  const int w_rows = kHalf >> p.div.tile[0].narrow;
  if (!make_map(&p.x, a.x, a.tokens, a.dim, a.x_row, kHalf) ||
      !make_map(&p.w[0], a.w_gate, a.hidden, a.dim, a.dim, w_rows) ||
      !make_map(&p.w[1], a.w_up, a.hidden, a.dim, a.dim, w_rows))
    return cudaErrorInvalidValue;
  uint16_t* out[3] = {a.h, a.g, a.u};
  p.save = a.g != nullptr;
  for (int i = 0; i < (p.save ? 3 : 1); ++i)
    if (!make_map(&p.out[i], out[i], a.tokens, a.hidden, a.hidden, kHalf))
      return cudaErrorInvalidValue;
  return a.act == kActSilu   ? launch_pairs<kActSilu>(p, pairs, a, stream)
         : a.act == kActGelu ? launch_pairs<kActGelu>(p, pairs, a, stream)
                             : launch_pairs<kActGeluTanh>(p, pairs, a, stream);
}

cudaError_t launch_ffn_bwd(const FfnBwdArgs& b, cudaStream_t stream) {
  const FfnArgs& a = b.f;
  const int64_t n = (int64_t)a.tokens * a.hidden / 8;
  const auto slope = a.act == kActSilu   ? slope_kernel<kActSilu>
                     : a.act == kActGelu ? slope_kernel<kActGelu>
                                         : slope_kernel<kActGeluTanh>;
  const cudaError_t e = launch_pdl(
      slope, dim3((unsigned)std::min<int64_t>((n + 255) / 256, a.sms * 8)),
      dim3(256), 0, stream, b);
  if (e != cudaSuccess) return e;
  PairParams p;
  memset(&p, 0, sizeof(p));
  const int kinds = b.dw_gate != nullptr ? 2 : 1;
  p.half_steps = up(a.hidden, kStep);
  int pairs;
  p.div = divide_bwd(a.tokens, a.dim, a.hidden, kinds == 2, a.sms, &pairs);
  const Tiles& dx = p.div.tile[p.div.kind[1] == kDx];
  const Tiles& dw = p.div.tile[p.div.kind[1] == kDw];
  const int64_t M = a.tokens, F = a.hidden, D = a.dim;
  p.dim_boxes = D % 64 == 0;
  p.hidden_boxes = F % 64 == 0;
  if (!make_column_map(&p.x, a.x, M, D, a.x_row, 2 - dw.narrow) ||
      !make_column_map(&p.w[0], a.w_gate, F, D, D, 2 - dx.narrow) ||
      !make_column_map(&p.w[1], a.w_up, F, D, D, 2 - dx.narrow) ||
      !make_map(&p.d[0], b.dg, M, F, F, kHalf) ||
      !make_map(&p.d[1], b.du, M, F, F, kHalf) ||
      !make_column_map(&p.dt[0], b.dg, M, F, F, 2) ||
      !make_column_map(&p.dt[1], b.du, M, F, F, 2))
    return cudaErrorInvalidValue;
  if (!make_map(&p.out[0], b.dx, a.tokens, a.dim, a.dim, kHalf) ||
      (kinds == 2 &&
       (!make_map(&p.out[1], b.dw_gate, a.hidden, a.dim, a.dim, kHalf) ||
        !make_map(&p.out[2], b.dw_up, a.hidden, a.dim, a.dim, kHalf))))
    return cudaErrorInvalidValue;
  return launch_pairs<-1>(p, pairs, a, stream);
}

}  // namespace fastvr
