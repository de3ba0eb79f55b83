// Attention of few query rows over the 4-bit cache: S = scale Q K^T,
// O = softmax(S) V with an online softmax in 32 bits, the codes expanded in
// registers.
//
// Bound by memory in principle: 0.5625 bytes per cached value, read once per
// block of query rows.  At the copy rate of the HBM an SM receives about 42
// values per clock, at about three issue slots each as written here, so the
// expansion has to be short and the products have to go to the tensor cores.
// Rows are too few for tcgen05 tiles (and the expanded operand would have to
// pass through shared memory): the expanded codes are the A operand of
// warp-level m16n8k16 products straight from registers, eight query rows the N
// side.
//
//   S^T[16 keys x 8 rows] = K[16 x d] Q^T     A: 16 keys of the cache
//   O^T[d x 8 rows] += V^T[d x 16] P^T        A: the transposed V block
//
// Expansion of K: a nibble y in the low bits of a half-precision float is the
// subnormal y 2^-24 (16 y 2^-24 one nibble up), which the tensor cores take as
// it is, so four logic operations and one shift expand eight codes and no
// arithmetic is left: Q, scaled by a power of two per row, is exact in half
// precision, the -8 of (y - 8) starts the accumulator as -8 sum q, and the
// group's scale multiplies its partial dot product in 32 bits.
//
// Expansion of V, whose scales lie along the contraction: a nibble y in bits
// 3..6 of a bfloat16 with the exponent of 16 is 16 + y (one shift and one
// logic operation for two of them), and one packed fused multiply-add gives
// (16 + y) s - 24 s = (y - 8) s, exact.
//
// The order of d inside a product is free as long as both operands share it.
// Lane (g, c) of a K fragment holds words 4 i + c of key row g for all groups
// i: one 16-byte piece of the stored row, whose words are permuted for this.
// A V fragment pairs two tokens in a register, so halves of two tokens' words
// are joined first; lane (g, c) holds d = 16 g .. 16 g + 15 (8 g .. 8 g + 7
// at d = 64), which lie in one scale group.  P leaves the first product with
// the keys on its rows and is turned by movmatrix into the second's operand.
// MMA row r of a block of 8 keys is key r / 2 + 4 (r % 2), so that the four
// token pairs that a V load touches lie in different banks.
//
// P enters its product as bfloat16 (2^-9 of each term): the values of the cache
// are exact in that type, not in half precision, whose exponent ends below
// theirs.  The row sum adds the unrounded P.  The output's relative error
// against 64 bits is 0.0019 to 0.0023; rounding the output alone leaves 0.0016
// to 0.0017.
//
// Measured (replayed from a graph): 604 MB of cache (8 streams of 65536 keys,
// 32 query heads over 8 key heads of 128) in 124 us, 4.9 TB/s; 906 MB (12 key
// heads) in 177 us, 5.1 TB/s.  In the steady state the integer pipe is busy for
// about 80 % of the cycles (logic, byte selection and moves of the expansion of
// V most of all), on average for 58 %; shifting V's nibbles by multiplication
// instead, on the other pipe, took 130 us, eight warps to an SM instead of
// sixteen 132.  One head and 4096 keys take 9.6 us, of which the stages that
// only one warp or CTA can do (its share, the first tile's way from memory, the
// join) are most.
//
// A warp streams its own key tiles (32 keys) through a ring in shared memory
// filled by cp.async, and keeps its own softmax state; the warps of a CTA and
// then the CTAs of a split key range are joined at the end, the latter by the
// CTA that finishes last (in a fixed order).  Keys outside the visible range
// are filled with zeros, scale included, so that whatever the cache holds
// there cannot reach the result.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "fastvr_internal.h"
#include "vec_math.cuh"

namespace fastvr {
namespace {

constexpr int kKeys = 32;         // keys of a warp's tile
constexpr float kThreshold = 8.f;  // log2 units, see chunk_attn_fwd.cu

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma_half(float (&c)[4], const uint32_t (&a)[4],
                                         uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
      "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4],
                                    uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
      "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Transpose of an 8 x 8 matrix of 16-bit elements held two per lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;"
               : "=r"(y)
               : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t scale_offset(uint32_t s) {  // -24 s, exact
  const __nv_bfloat162 v =
      __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&s),
              __floats2bfloat162_rn(-24.f, -24.f));
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Nibbles J and J + 4 of w as two bfloat16 values, with scale and offset.
template <int J>
__device__ __forceinline__ uint32_t expand(uint32_t w, uint32_t s, uint32_t o) {
  const uint32_t x = J == 0 ? w << 3 : w >> (J == 0 ? 0 : 4 * J - 3);
  const uint32_t m = (x & 0x00780078u) | 0x41804180u;
  const __nv_bfloat162 v =
      __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&m),
              *reinterpret_cast<const __nv_bfloat162*>(&s),
              *reinterpret_cast<const __nv_bfloat162*>(&o));
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int D>
struct Tile {  // one stage of a warp's ring, byte offsets
  static constexpr int kRow = D / 2;       // bytes of a row of codes
  static constexpr int kScale = D / 16;    // bytes of a row of scales
  static constexpr int k = 0;
  static constexpr int v = kKeys * kRow;
  static constexpr int ks = 2 * kKeys * kRow;
  static constexpr int vs = ks + kKeys * kScale;
  static constexpr int bytes = vs + kKeys * kScale;
};

// Byte offset of 8-byte piece x of row r of a V tile: at d = 128 the halves
// of rows 2, 3, 6, 7, ... are swapped, so that the 8-byte loads of a half
// warp (4 tokens x 4 pieces) touch every bank once.
template <int D>
__device__ __forceinline__ int v_offset(int r, int byte) {
  return r * Tile<D>::kRow + (D == 128 ? byte ^ ((r & 2) << 4) : byte);
}

// A unit is a block of query rows of one key head of one batch entry.  The
// tiles of all units laid end to end (row blocks fastest, batch entries
// slowest) are cut into even shares, one to a CTA, however different the
// entries' lengths are.  Every unit counts kUnitCost tiles more than it has,
// about what starting and ending it costs, so that a CTA with many short
// units is not the last one (eight streams of 6000 to 66000 keys: 64.7 us with
// 12, 57.0 with 24, 58.1 with 32); an entry that sees no key still has units,
// whose zeros someone writes.
constexpr int kUnitCost = 24;

// A CTA's part of a unit.
struct Piece {
  bool more;           // there is one
  int b, hk, rb;
  int first, j0, j1;   // first visible key; tiles [j0, j1) of the unit
  // The CTAs that share the unit are cta0 .. cta0 + parts - 1.  Each has two
  // slots for partial results, 0 for the unit that its share begins in and 1
  // for the one that it ends in.  cta0 uses slot0, the others 0, this CTA
  // `mine`.  Of the units that begin in a CTA only the last one goes on in
  // others, so that cta0's ticket counts the unit's parts.
  int cta0, parts, slot0, mine;
};

template <int NT, int W, int kGroups>
struct Shared {
  float m[W][8 * NT], l[W][8 * NT];
  float start[kGroups][8 * NT];  // first value of a dot product
  uint4 q[NT > 1 ? NT : 1][NT > 1 ? kGroups : 1][32];
  Piece piece[2];       // this one and the next
  Piece shared[2];      // by slot: the units that other CTAs have parts of
  int64_t total, at;    // counted tiles in all; the share's next one
  int64_t before;       // counted tiles of the entries before b
  int ctas, b;          // CTAs that have a share
  int last[2];          // this CTA joins the parts of shared[i]
};

// a / b; in 32 bits, many times faster, where both fit
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

__device__ __forceinline__ int first_key(const Q4AttnParams& p, int b) {
  return p.first_chunk == nullptr
             ? 0
             : (int)first_visible_token(p.first_chunk[b], p.lo_chunk,
                                        p.chunk_tokens, p.keys);
}
__device__ __forceinline__ int tiles_from(const Q4AttnParams& p, int first) {
  return ((int)p.keys - first + kKeys - 1) / kKeys;
}

// Warp 0: the counted tiles of the launch and the entry that this CTA's share
// begins in.
template <class S>
__device__ void find_share(const Q4AttnParams& p, S* sh) {
  const int lane = threadIdx.x % 32;
  const int units_b = p.kv_heads * p.row_blocks;  // units of a batch entry
  auto counted = [&](int b) -> int64_t {
    return b < p.batch
               ? (int64_t)(tiles_from(p, first_key(p, b)) + kUnitCost) * units_b
               : 0;
  };
  int64_t total = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    int64_t n = counted(b0 + lane);
#pragma unroll
    for (int y = 16; y > 0; y /= 2) n += __shfl_xor_sync(0xffffffffu, n, y);
    total += n;
  }
  // no more CTAs than tiles: an empty share inside a unit would leave its
  // ticket short of a part
  const int ctas = (int)min((int64_t)gridDim.x, total);
  const int64_t begin = divide(total * blockIdx.x, ctas);
  int64_t before = 0;
  int b = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int64_t n = counted(b0 + lane);
    int64_t sum = n;  // inclusive
#pragma unroll
    for (int y = 1; y < 32; y *= 2) {
      const int64_t v = __shfl_up_sync(0xffffffffu, sum, y);
      if (lane >= y) sum += v;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, before + sum > begin);
    if (past != 0) {
      const int i = __ffs(past) - 1;
      before += __shfl_sync(0xffffffffu, sum - n, i);
      b = b0 + i;
      break;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (lane == 0) {
    sh->total = total;
    sh->ctas = ctas;
    sh->at = begin;
    sh->before = before;
    sh->b = b;
  }
}

// Thread 0: the share's next piece.
template <class S>
__device__ __noinline__ void next_piece(const Q4AttnParams& p, S* sh,
                                        Piece* out) {
  const int ctas = sh->ctas;
  const int64_t total = sh->total, at = sh->at;
  const int64_t begin = divide(total * blockIdx.x, ctas);
  const int64_t end = divide(total * (blockIdx.x + 1), ctas);
  out->more = (int)blockIdx.x < ctas && at < end;
  if (!out->more) return;
  const int units_b = p.kv_heads * p.row_blocks;
  int b = sh->b;
  int64_t before = sh->before;
  int first = first_key(p, b);
  int count = tiles_from(p, first) + kUnitCost;
  while (at >= before + (int64_t)count * units_b) {
    before += (int64_t)count * units_b;
    ++b;
    first = first_key(p, b);
    count = tiles_from(p, first) + kUnitCost;
  }
  const int in_b = (int)divide(at - before, count);
  const int64_t unit0 = before + (int64_t)in_b * count;
  out->b = b;
  out->rb = in_b % p.row_blocks;
  out->hk = in_b / p.row_blocks;
  out->first = first;
  // the first kUnitCost counted tiles have no keys
  out->j0 = max(0, (int)(at - unit0) - kUnitCost);
  out->j1 = max(0, (int)min((int64_t)count, end - unit0) - kUnitCost);
  const int cta0 = (int)divide((unit0 + 1) * ctas - 1, total);
  out->cta0 = cta0;
  out->parts = (int)divide((unit0 + count) * ctas - 1, total) - cta0 + 1;
  out->slot0 = divide(total * cta0, ctas) == unit0 ? 0 : 1;
  out->mine = at == begin ? 0 : 1;
  sh->b = b;
  sh->before = before;
  sh->at = min(end, unit0 + count);
}

// Partial results: O (for its own m) [CTA][slot][row][D] and, behind all of
// them, m and l [CTA][slot][row].
template <int D>
__device__ __forceinline__ float2* partial_ml(const Q4AttnParams& p) {
  return reinterpret_cast<float2*>(p.partial +
                                   (int64_t)kQ4MaxParts * kQ4PartRows * D);
}

// Four columns of a row of a unit, from the sums over all its keys.
template <int D, int kRows>
__device__ __forceinline__ void finish(const Q4AttnParams& p,
                                       const Piece& piece, int row, int d,
                                       float4 acc, float sum, float top) {
  const int r = piece.rb * kRows + row;
  const int tok = r / p.group, head = piece.hk * p.group + r % p.group;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;  // no key: zeros
  *reinterpret_cast<uint2*>(
      p.out +
      (((int64_t)piece.b * p.q_tokens + tok) * p.heads + head) * D + d) =
      make_uint2(pack(acc.x * inv, acc.y * inv),
                 pack(acc.z * inv, acc.w * inv));
  if (d == 0 && p.lse != nullptr)
    p.lse[((int64_t)piece.b * p.heads + head) * p.q_tokens + tok] =
        sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

// The end of a piece: joins the warps' results (m and l in sh, O[row][d] for
// its own m in each warp's part of `smem`) into the output, or into a partial
// result when other CTAs have parts of the unit.
template <int D, int NT, int W, int kWarpBytes, class S>
__device__ __forceinline__ void end_piece(const Q4AttnParams& p, S* sh,
                                          const uint8_t* smem,
                                          const Piece& piece) {
  constexpr int kRows = 8 * NT;
  constexpr int kPitch = D + 4;
  const int rows = min(kRows, p.rows - piece.rb * kRows);
  const int part = ((int)blockIdx.x * 2 + piece.mine) * kRows;
  // A thread takes 4 columns of a row.
  constexpr int kSlots = D / 4;
  const int slots = rows * kSlots;
  for (int x = threadIdx.x; x < slots; x += W * 32) {
    const int row = x / kSlots, d = x % kSlots * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, sh->m[w][row]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      // a warp without keys (m = -inf, l = 0) adds nothing
      const float mw = sh->m[w][row], lw = sh->l[w][row];
      const float f = mw == -INFINITY && lw == 0.f ? 0.f : ex2(mw - top);
      const float4 v = *reinterpret_cast<const float4*>(
          smem + w * kWarpBytes + (row * kPitch + d) * 4);
      acc.x = fmaf(f, v.x, acc.x);
      acc.y = fmaf(f, v.y, acc.y);
      acc.z = fmaf(f, v.z, acc.z);
      acc.w = fmaf(f, v.w, acc.w);
      sum = fmaf(f, lw, sum);
    }
    if (piece.parts == 1) {
      finish<D, kRows>(p, piece, row, d, acc, sum, top);
    } else {
      *reinterpret_cast<float4*>(p.partial + (int64_t)(part + row) * D + d) =
          acc;
      if (d == 0) partial_ml<D>(p)[part + row] = make_float2(top, sum);
    }
  }
  if (threadIdx.x == 0 && piece.parts > 1) sh->shared[piece.mine] = piece;
}

// The last CTA of a unit to arrive joins its parts, in their order: m and l of
// all of them first, the weight of every (part, row) from these, then sums of
// weighted rows.  Each step has its loads in flight together: what a join costs
// is their latency (32 rows over 4096 keys of 12 heads: 25.5 us with a row and
// a few loads at a time, 21.8 now).
template <int D, int NT, int W, int kWarpBytes, class S>
__device__ __forceinline__ void join_parts(const Q4AttnParams& p, S* sh,
                                           uint8_t* smem, const Piece& piece) {
  constexpr int kRows = 8 * NT, kThreads = W * 32;
  int tid;  // read anew: what follows from it is not kept across the tiles
  asm volatile("mov.u32 %0, %%tid.x;" : "=r"(tid));
  const int warp = tid / 32, lane = tid % 32;
  const int parts = piece.parts, cta0 = piece.cta0, slot0 = piece.slot0;
  const int rows = min(kRows, p.rows - piece.rb * kRows);
  auto slot_of = [&](int cta) {
    return (cta * 2 + (cta == cta0 ? slot0 : 0)) * kRows;
  };
  const float2* all_ml = partial_ml<D>(p);
  constexpr int kPitch = kRows + 1;
  float2* ml = reinterpret_cast<float2*>(smem);  // [part][row]
  constexpr int kAtOnce = 32 / kRows;            // parts to a warp
  const int r = lane % kRows;
#pragma unroll 4
  for (int i = warp * kAtOnce + lane / kRows; i < parts; i += W * kAtOnce)
    if (r < rows) ml[i * kPitch + r] = __ldcg(all_ml + slot_of(cta0 + i) + r);
  __syncthreads();
  // Rows warp, warp + W, ... of a warp, side by side.
  constexpr int kOwn = (kRows + W - 1) / W;
  float top[kOwn], sum[kOwn];
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    top[k] = -INFINITY;
    sum[k] = 0.f;
  }
  for (int i = lane; i < parts; i += 32)
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      if (warp + k * W < rows)
        top[k] = fmaxf(top[k], ml[i * kPitch + warp + k * W].x);
#pragma unroll
  for (int y = 16; y > 0; y /= 2)
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], y));
  for (int i = lane; i < parts; i += 32)
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      if (warp + k * W < rows) {
        float2& v = ml[i * kPitch + warp + k * W];
        // a part without keys has m = -inf and l = 0
        const float f =
            v.x == -INFINITY && v.y == 0.f ? 0.f : ex2(v.x - top[k]);
        v.x = f;
        sum[k] = fmaf(f, v.y, sum[k]);
      }
#pragma unroll
  for (int y = 16; y > 0; y /= 2)
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], y);
  if (lane < kOwn && warp + lane * W < rows) {
    // lane k: row warp + k W
    float m = top[0], l = sum[0];
#pragma unroll
    for (int k = 1; k < kOwn; ++k)
      if (lane == k) m = top[k], l = sum[k];
    const int row = warp + lane * W;
    sh->m[0][row] = m;
    sh->l[0][row] = l;
  }
  __syncthreads();
  // A thread takes up to kPer pieces of 4 columns; with few rows the parts are
  // shared out over `share` threads, whose sums are added in their order.
  constexpr int kSlots = D / 4;
  constexpr int kPer = (kRows * kSlots + kThreads - 1) / kThreads;
  constexpr int kBatch = NT == 1 ? 8 : 16 / kPer;
  const int slots = rows * kSlots;
  static_assert(kQ4MaxCtas * kPitch * 8 + kThreads * 16 <= W * kWarpBytes,
                "weights and sums do not fit");
  float4* sums = reinterpret_cast<float4*>(ml + kQ4MaxCtas * kPitch);
  const int share = max(1, kThreads / slots);
  const int who = share > 1 ? tid / slots : 0;
  const int x0 = tid - who * slots;
  float4 acc[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (who < share)
    for (int i0 = who; i0 < parts; i0 += kBatch * share) {
      float4 v[kPer][kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (i0 + u * share < parts) {
          const float* src = p.partial + slot_of(cta0 + i0 + u * share) * D;
#pragma unroll
          for (int k = 0; k < kPer; ++k)
            if (x0 + k * kThreads < slots)
              v[k][u] = __ldcg(
                  reinterpret_cast<const float4*>(src) + x0 + k * kThreads);
        }
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (i0 + u * share < parts)
#pragma unroll
          for (int k = 0; k < kPer; ++k)
            if (x0 + k * kThreads < slots) {
              const float f = ml[(i0 + u * share) * kPitch +
                                 (x0 + k * kThreads) / kSlots].x;
              acc[k].x = fmaf(f, v[k][u].x, acc[k].x);
              acc[k].y = fmaf(f, v[k][u].y, acc[k].y);
              acc[k].z = fmaf(f, v[k][u].z, acc[k].z);
              acc[k].w = fmaf(f, v[k][u].w, acc[k].w);
            }
    }
  if (share > 1) {
    sums[tid] = acc[0];
    __syncthreads();
    if (who == 0)
      for (int i = 1; i < share; ++i) {
        if (x0 >= slots) break;
        const float4 v = sums[i * slots + x0];
        acc[0].x += v.x, acc[0].y += v.y, acc[0].z += v.z, acc[0].w += v.w;
      }
  }
  if (who == 0)
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int x = x0 + k * kThreads, row = x / kSlots;
      if (x < slots)
        finish<D, kRows>(p, piece, row, x % kSlots * 4, acc[k], sh->l[0][row],
                         sh->m[0][row]);
    }
}

// NT blocks of 8 query rows, W warps, kStages tiles in each warp's ring, kCtas
// CTAs to an SM.
template <int D, int NT, int W, int kStages, int kCtas>
__global__ void __launch_bounds__(W * 32, kCtas)
q4_attn_kernel(const __grid_constant__ Q4AttnParams p) {
  using L = Tile<D>;
  constexpr int kGroups = D / 32;
  constexpr int kWords = D / 64;  // V words (8 values) of a lane per token
  constexpr bool kQShared = NT > 1;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Shared<NT, W, kGroups> sh;
  pdl_trigger();
  pdl_wait();
  if (threadIdx.x < 32) find_share(p, &sh);
  if (threadIdx.x < 2) sh.shared[threadIdx.x].parts = 1;
  if (threadIdx.x == 0) next_piece(p, &sh, &sh.piece[0]);
  __syncthreads();

  const int keys = (int)p.keys;
  const uint32_t cache_tokens = (uint32_t)p.cache_tokens;
  for (int k = 0;; k ^= 1) {
    const Piece* piece = &sh.piece[k];
    if (!piece->more) break;
    // read anew for every unit: what follows from it is then not kept in
    // registers across the end of the previous one
    int tid;
    asm volatile("mov.u32 %0, %%tid.x;" : "=r"(tid));
    const int warp = tid / 32, lane = tid % 32;
    const int g = lane / 4, c = lane % 4;
    uint8_t* ring = smem + warp * kStages * L::bytes;
    const uint32_t ring_u = smem_u32(ring);
    const int b = piece->b, hk = piece->hk, rb = piece->rb;
    const int first = piece->first, j0 = piece->j0, j1 = piece->j1;
    // bytes of codes before this head's; its scales take an eighth as many
    const int64_t head_at =
        ((int64_t)b * p.kv_heads + hk) * p.cache_tokens * L::kRow;
    static_assert(L::kRow == 8 * L::kScale, "");

    constexpr int kPieces = L::kRow / 16;  // 16-byte pieces of a row
    // This lane's piece of every 32 / kPieces rows of a tile.
    const uint32_t k_dst = ring_u + L::k + lane * 16;
    const uint32_t v_dst =
        ring_u + L::v + v_offset<D>(lane / kPieces, lane % kPieces * 16);
    const uint32_t s_dst = ring_u + L::ks + lane * L::kScale;
    auto fetch = [&](int j, int stage) {
      if (j < j1) {
        const int key0 = first + j * kKeys;
        uint32_t row0 = (uint32_t)p.first_row + key0;  // both below 2^30
        if (row0 >= cache_tokens) row0 -= cache_tokens;
        const uint32_t to = stage * L::bytes;
        if (key0 + kKeys <= keys && row0 + kKeys <= cache_tokens) {
          // the usual tile: 32 rows in one piece
          const int64_t at = head_at + (int64_t)row0 * L::kRow + lane * 16;
          const uint8_t* kc = p.k_codes + at;
          const uint8_t* vc = p.v_codes + at;
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            copy_async<16>(k_dst + to + i * 512, kc + i * 512, true);
            copy_async<16>(v_dst + to + i * 512, vc + i * 512, true);
          }
          const int64_t st =
              head_at / 8 + (int64_t)(row0 + lane) * L::kScale;
          copy_async<L::kScale>(s_dst + to, p.k_scales + st, true);
          copy_async<L::kScale>(s_dst + to + L::vs - L::ks, p.v_scales + st,
                                true);
        } else {
          auto cache_row = [&](int r) {
            const uint32_t x = row0 + r;
            return (int64_t)(x >= cache_tokens ? x - cache_tokens : x);
          };
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            const int r = (i * 32 + lane) / kPieces;
            const bool ok = key0 + r < keys;
            const int64_t at = head_at + (ok ? cache_row(r) : 0) * L::kRow +
                               lane % kPieces * 16;
            copy_async<16>(k_dst + to + i * 512, p.k_codes + at, ok);
            copy_async<16>(v_dst + to + i * 512, p.v_codes + at, ok);
          }
          const bool ok = key0 + lane < keys;
          const int64_t st =
              head_at / 8 + (ok ? cache_row(lane) : 0) * L::kScale;
          copy_async<L::kScale>(s_dst + to, p.k_scales + st, ok);
          copy_async<L::kScale>(s_dst + to + L::vs - L::ks, p.v_scales + st,
                                ok);
        }
      }
      copy_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(j0 + warp + s * W, s);

    // Q^T fragments in half precision: for group i, element pairs (e, e + 4) of
    // words 4 i + c, those of odd e divided by 16 (their codes lie one nibble
    // up), all times the power of two that brings the row's largest magnitude
    // to [2^15, 2^16) (of magnitudes up to 2^100).
    // All warps need the same ones: with more than one block they stay in
    // shared memory, which leaves their registers to the sums.
    uint32_t qf[kQShared ? 1 : NT][kGroups][4];
    float unit[NT][2];  // score of a dot product of 1, rows 2 c and 2 c + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = (rb * NT + nt) * 8 + g;
      const int tok = row / p.group, head = hk * p.group + row % p.group;
      const uint16_t* q =
          p.q + (((int64_t)b * p.q_tokens + tok) * p.heads + head) * D;
      uint4 w[kGroups];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        w[i] = make_uint4(0, 0, 0, 0);
        if (row < p.rows)
          w[i] = *reinterpret_cast<const uint4*>(q + 32 * i + 8 * c);
        const uint32_t m = 0x7fff7fffu;
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(w[i].x & m, w[i].y & m),
                                     __vmaxu2(w[i].z & m, w[i].w & m)));
      }
      top = max(top >> 16, top & 0xffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // exponent of the largest magnitude, kept where powers of two stay finite
      const int e = min(max((int)(top >> 7) - 127, -100), 100);
      const float up = __int_as_float((15 - e + 127) << 23);
      // 2^24 of the subnormal codes, 2^(e - 15) of the row
      const float mine = p.scale_log2 * __int_as_float((24 - 15 + e + 127) << 23);
      unit[nt][0] = __shfl_sync(0xffffffffu, mine, 8 * c);
      unit[nt][1] = __shfl_sync(0xffffffffu, mine, 8 * c + 4);
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        float f[8], sum = 0.f;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          f[2 * y] = __uint_as_float(x[y] << 16) * up;
          f[2 * y + 1] = __uint_as_float(x[y] & 0xffff0000u) * up;
          sum += f[2 * y] + f[2 * y + 1];
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float k = y % 2 ? 0.0625f : 1.f;
          const __half2 h = __floats2half2_rn(f[y] * k, f[y + 4] * k);
          qf[kQShared ? 0 : nt][i][y] = *reinterpret_cast<const uint32_t*>(&h);
        }
        if (kQShared && warp == 0)
          sh.q[nt][i][lane] = make_uint4(qf[0][i][0], qf[0][i][1], qf[0][i][2],
                                        qf[0][i][3]);
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (warp == 0 && c == 0) sh.start[i][nt * 8 + g] = sum * (-8.f * 0x1p-24f);
      }
    }
    if (tid == 0) next_piece(p, &sh, &sh.piece[k ^ 1]);
    __syncthreads();

    float o[NT][D / 16][4];
    float m[NT][2], l[NT][2];  // rows 2 c and 2 c + 1 of each block
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
    }

    int stage = 0;
    const int kr = (g >> 1) + (g & 1) * 4;  // key of MMA row g
    for (int j = j0 + warp; j < j1; j += W) {
      copy_wait<kStages - 2>();
      __syncwarp();
      {
        int ahead = stage + kStages - 1;
        if (ahead >= kStages) ahead -= kStages;
        fetch(j + (kStages - 1) * W, ahead);
      }
      const uint8_t* t = ring + stage * L::bytes;
      if (++stage == kStages) stage = 0;

      // S^T: two blocks of 16 keys, in units of `unit`
      float s[NT][2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t w[2][kGroups];
        float sc[2][kGroups];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int r = x * 16 + y * 8 + kr;
          if constexpr (D == 128) {
            const uint4 v = *reinterpret_cast<const uint4*>(t + L::k +
                                                            r * L::kRow + c * 16);
            w[y][0] = v.x, w[y][1] = v.y, w[y][2] = v.z, w[y][3] = v.w;
            const uint2 f =
                *reinterpret_cast<const uint2*>(t + L::ks + r * L::kScale);
            sc[y][0] = __uint_as_float(f.x << 16);
            sc[y][1] = __uint_as_float(f.x & 0xffff0000u);
            sc[y][2] = __uint_as_float(f.y << 16);
            sc[y][3] = __uint_as_float(f.y & 0xffff0000u);
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(t + L::k +
                                                            r * L::kRow + c * 8);
            w[y][0] = v.x, w[y][1] = v.y;
            const uint32_t f =
                *reinterpret_cast<const uint32_t*>(t + L::ks + r * L::kScale);
            sc[y][0] = __uint_as_float(f << 16);
            sc[y][1] = __uint_as_float(f & 0xffff0000u);
          }
        }
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const uint32_t lo = 0x000f000fu, hi = 0x00f000f0u;
          const uint32_t u0 = w[0][i] >> 8, u1 = w[1][i] >> 8;
          const uint32_t a0[4] = {w[0][i] & lo, w[1][i] & lo, w[0][i] & hi,
                                  w[1][i] & hi};
          const uint32_t a1[4] = {u0 & lo, u1 & lo, u0 & hi, u1 & hi};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float2 z =
                *reinterpret_cast<const float2*>(&sh.start[i][nt * 8 + 2 * c]);
            float d[4] = {z.x, z.y, z.x, z.y};
            const uint32_t(&r)[4] = qf[kQShared ? 0 : nt][i];
            const uint4 q = kQShared ? sh.q[kQShared ? nt : 0][i][lane]
                                     : make_uint4(r[0], r[1], r[2], r[3]);
            mma_half(d, a0, q.x, q.y);
            mma_half(d, a1, q.z, q.w);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[nt][x][e] = i == 0 ? d[e] * sc[e / 2][i]
                                   : fmaf(d[e], sc[e / 2][i], s[nt][x][e]);
          }
        }
      }

      // Softmax over the tile's 32 keys; lane: keys x 16 + e/2 8 + kr of rows
      // 2 c + e % 2.
      const int left = keys - first - j * kKeys;
      if (left < kKeys) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (x * 16 + (e / 2) * 8 + kr >= left) s[nt][x][e] = -INFINITY;
      }
      uint32_t pt[NT][2][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          top[q] = fmaxf(fmaxf(s[nt][0][q], s[nt][0][q + 2]),
                         fmaxf(s[nt][1][q], s[nt][1][q + 2]));
#pragma unroll
          for (int y = 4; y < 32; y *= 2)
            top[q] = fmaxf(top[q], __shfl_xor_sync(0xffffffffu, top[q], y));
          top[q] *= unit[nt][q];
        }
        if (__any_sync(0xffffffffu, top[0] > m[nt][0] + kThreshold ||
                                        top[1] > m[nt][1] + kThreshold)) {
          float f[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float mn = fmaxf(m[nt][q], top[q]);
            f[q] = mn == -INFINITY ? 1.f : ex2(m[nt][q] - mn);
            l[nt][q] *= f[q];
            m[nt][q] = mn;
          }
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][i][e] *= f[e % 2];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[nt][x][e] =
                ex2(fmaf(s[nt][x][e], unit[nt][e % 2], -m[nt][e % 2]));
            l[nt][e % 2] += s[nt][x][e];
          }
          pt[nt][x][0] = transpose8(pack(s[nt][x][0], s[nt][x][1]));
          pt[nt][x][1] = transpose8(pack(s[nt][x][2], s[nt][x][3]));
        }
      }

      // O^T += V^T P^T: MMA column pairs of block x are tokens c, c + 4 and
      // 8 + c, 12 + c.
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t w[4][kWords], sv[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int r = x * 16 + y * 4 + c;
          if constexpr (D == 128) {
            const uint2 v = *reinterpret_cast<const uint2*>(
                t + L::v + v_offset<D>(r, g * 8));
            w[y][0] = v.x, w[y][1] = v.y;
          } else {
            w[y][0] = *reinterpret_cast<const uint32_t*>(t + L::v + r * L::kRow +
                                                         g * 4);
          }
          // the group of this lane's elements: 16 g / 32 or 8 g / 32
          sv[y] = *reinterpret_cast<const uint16_t*>(
              t + L::vs + r * L::kScale + (D == 128 ? g / 2 : g / 4) * 2);
        }
        const uint32_t s0 = sv[0] | (sv[1] << 16), s1 = sv[2] | (sv[3] << 16);
        const uint32_t o0 = scale_offset(s0), o1 = scale_offset(s1);
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
          // (token pair 0 | 1) x (elements 0..3 | 4..7)
          const uint32_t a00 = __byte_perm(w[0][i], w[1][i], 0x5410);
          const uint32_t a01 = __byte_perm(w[0][i], w[1][i], 0x7632);
          const uint32_t a10 = __byte_perm(w[2][i], w[3][i], 0x5410);
          const uint32_t a11 = __byte_perm(w[2][i], w[3][i], 0x7632);
#define FASTVR_PV(J)                                                  \
  {                                                                   \
    const uint32_t a[4] = {expand<J>(a00, s0, o0), expand<J>(a01, s0, o0), \
                           expand<J>(a10, s1, o1), expand<J>(a11, s1, o1)}; \
    _Pragma("unroll") for (int nt = 0; nt < NT; ++nt)                 \
        mma(o[nt][4 * i + J], a, pt[nt][x][0], pt[nt][x][1]);         \
  }
          FASTVR_PV(0) FASTVR_PV(1) FASTVR_PV(2) FASTVR_PV(3)
#undef FASTVR_PV
        }
      }
    }
    copy_wait<0>();
    __syncwarp();

    // Each warp leaves m, l and O[row][d] (for its own m) in shared memory.
    float* so = reinterpret_cast<float*>(ring);
    constexpr int kPitch = D + 4;
    static_assert(8 * NT * kPitch * 4 <= kStages * L::bytes, "ring too small");
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float x = l[nt][q];
#pragma unroll
        for (int y = 4; y < 32; y *= 2) x += __shfl_xor_sync(0xffffffffu, x, y);
        const int row = nt * 8 + 2 * c + q;
        if (g == 0) {
          sh.m[warp][row] = m[nt][q];
          sh.l[warp][row] = x;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            *reinterpret_cast<float4*>(so + row * kPitch + 8 * kWords * g +
                                       8 * i + 4 * y) =
                make_float4(o[nt][4 * i][2 * y + q], o[nt][4 * i + 1][2 * y + q],
                            o[nt][4 * i + 2][2 * y + q],
                            o[nt][4 * i + 3][2 * y + q]);
      }
    __syncthreads();
    end_piece<D, NT, W, kStages * L::bytes>(p, &sh, smem, *piece);
    __syncthreads();  // before the next unit's tiles and the piece after it
  }

  // Of the units that this CTA shares with others it joins those whose last
  // part it was.
  __threadfence();
  __syncthreads();
  if (threadIdx.x < 2) {
    const Piece& mine = sh.shared[threadIdx.x];
    bool last = false;
    if (mine.parts > 1) {
      last = atomicAdd(p.tickets + mine.cta0, 1) == mine.parts - 1;
      if (last) p.tickets[mine.cta0] = 0;  // for the next call
    }
    sh.last[threadIdx.x] = last;
  }
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    if (!sh.last[i]) continue;
    __threadfence();
    join_parts<D, NT, W, kStages * L::bytes>(p, &sh, smem, sh.shared[i]);
    __syncthreads();
  }
}

template <int D, int NT, int kWarps, int kStages, int kCtas>
cudaError_t launch_v(Q4AttnParams p, int sms, cudaStream_t stream) {
  p.row_blocks = (p.rows + 8 * NT - 1) / (8 * NT);
  const int64_t units = (int64_t)p.batch * p.kv_heads * p.row_blocks;
  const int64_t tiles = units * ((p.keys + kKeys - 1) / kKeys + kUnitCost);
  // Either as many CTAs as the SMs hold at once, sharing out the tiles whatever
  // the units, or the same number to every unit (no CTA then has more than one
  // piece when the entries are equally long): whichever has the shortest
  // estimated time in clocks, a round of tiles (each warp one) taking about
  // 1000 with 8 query rows and half as much for every further 8, a piece 3000,
  // and the join of a unit 2000 and its bytes at 64 per clock.
  const int64_t rows = std::min(p.rows, 8 * NT);
  const int64_t slots = std::min(sms * kCtas, kQ4MaxCtas);
  int64_t grid = slots, best = INT64_MAX;
  auto consider = [&](int64_t n, int64_t pieces, int64_t parts) {
    const int64_t rounds = (tiles + n * kWarps - 1) / (n * kWarps);
    const int64_t cost = rounds * 500 * (NT + 1) + pieces * 3000 +
                         (parts > 1 ? 2000 + parts * rows * D / 16 : 0);
    if (cost < best) {
      best = cost;
      grid = n;
    }
  };
  for (int64_t parts = 1; parts * units <= slots; ++parts)
    consider(parts * units, 1, parts);
  consider(slots, (units + slots - 1) / slots + 1, (slots + units - 1) / units + 1);
  constexpr int smem = kWarps * kStages * Tile<D>::bytes;
  auto kernel = q4_attn_kernel<D, NT, kWarps, kStages, kCtas>;
  const cudaError_t e = cudaFuncSetAttribute(
      kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(kWarps * 32), smem,
                    stream, p);
}

template <int D>
cudaError_t launch_d(const Q4AttnParams& p, int sms, cudaStream_t stream) {
  // Warps and ring depths are what registers and shared memory hold: 16 warps
  // of 128 registers with one block of rows, 8 with two (16 rows over 65536
  // keys of 12 heads: 46.8 us; 10 warps spill, 52.0) or four.  With four at
  // d = 128 the eight spill some all the same (368 bytes stored, 312 loaded).
  constexpr int kDeep = D == 128 ? 1 : 2;
  if (p.rows <= 8) return launch_v<D, 1, 8, 3 * kDeep, 2>(p, sms, stream);
  if (p.rows <= 16) return launch_v<D, 2, 8, 4 * kDeep, 1>(p, sms, stream);
  return launch_v<D, 4, 8, 4 * kDeep, 1>(p, sms, stream);
}

}  // namespace

cudaError_t launch_q4_attn(const Q4AttnParams& p, int sms,
                           cudaStream_t stream) {
  if (p.head_dim == 64) return launch_d<64>(p, sms, stream);
  if (p.head_dim == 128) return launch_d<128>(p, sms, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastvr
