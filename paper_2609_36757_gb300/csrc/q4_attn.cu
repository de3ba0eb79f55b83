// Attention of few query rows over the 4-bit cache: S = scale Q K^T,
// O = softmax(S) V with an online softmax in 32 bits, the codes expanded in
// registers.
//
// Bound by memory: 0.5625 bytes per cached value, read once per block of
// query rows.  At the copy rate of the HBM an SM receives about 42 values per
// clock, three issue slots each, so the expansion has to be short and the
// products have to go to the tensor cores.  Rows are too few for tcgen05
// tiles (and the expanded operand would have to pass through shared memory):
// the expanded codes are the A operand of warp-level m16n8k16 products
// straight from registers, eight query rows the N side.
//
//   S^T[16 keys x 8 rows] = K[16 x d] Q^T     A: 16 keys of the cache
//   O^T[d x 8 rows] += V^T[d x 16] P^T        A: the transposed V block
//
// A nibble y is placed in bits 3..6 of a bfloat16 with the exponent of 16
// (one shift, one logic operation for two of them), which is 16 + y, and one
// packed fused multiply-add gives (16 + y) s - 24 s = (y - 8) s, exact.
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
// A warp streams its own key tiles (32 keys) through a ring in shared memory
// filled by cp.async, and keeps its own softmax state; the warps of a CTA and
// then the CTAs of a split key range are joined at the end, the latter by the
// CTA that finishes last (in a fixed order).  Keys outside the visible range
// are filled with zeros, scale included, so that whatever the cache holds
// there cannot reach the result.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

constexpr int kKeys = 32;         // keys of a warp's tile
constexpr float kThreshold = 8.f;  // log2 units, see chunk_attn_fwd.cu

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// Asynchronous copy of N bytes to shared memory, zeros when !valid.
template <int N>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src,
                                           bool valid) {
  const int n = valid ? N : 0;
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst),
                 "l"(src), "r"(n)
                 : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst),
                 "l"(src), "n"(N), "r"(n)
                 : "memory");
}
__device__ __forceinline__ void copy_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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

// NT blocks of 8 query rows, W warps, kStages tiles in each warp's ring.
template <int D, int NT, int W, int kStages>
__global__ void __launch_bounds__(W * 32)
q4_attn_kernel(const __grid_constant__ Q4AttnParams p) {
  using L = Tile<D>;
  constexpr int kGroups = D / 32;
  constexpr int kWords = D / 64;  // V words (8 values) of a lane per token
  constexpr int kRows = 8 * NT;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_m[W][kRows], s_l[W][kRows];
  __shared__ int s_last;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int g = lane / 4, c = lane % 4;
  uint8_t* ring = smem + warp * kStages * L::bytes;
  const uint32_t ring_u = smem_u32(ring);

  // This CTA: key range `split` of row block rb of (b, kv head).
  const int rb = blockIdx.x % p.row_blocks;
  const int bh = blockIdx.x / p.row_blocks % p.batch_heads;
  const int split = blockIdx.x / p.row_blocks / p.batch_heads;
  const int b = bh / p.kv_heads, hk = bh % p.kv_heads;
  pdl_trigger();
  pdl_wait();

  // Logical keys are counted from the oldest chunk of the window.
  const int64_t first =
      p.first_chunk == nullptr
          ? 0
          : first_visible_token(p.first_chunk[b], p.lo_chunk, p.chunk_tokens,
                                p.keys);
  const int64_t tiles = (p.keys - first + kKeys - 1) / kKeys;
  const int64_t j0 = tiles * split / p.splits;
  const int64_t j1 = tiles * (split + 1) / p.splits;

  const uint8_t* k_codes =
      p.k_codes + (int64_t)bh * p.cache_tokens * L::kRow;
  const uint8_t* v_codes =
      p.v_codes + (int64_t)bh * p.cache_tokens * L::kRow;
  const uint8_t* k_scales =
      p.k_scales + (int64_t)bh * p.cache_tokens * L::kScale;
  const uint8_t* v_scales =
      p.v_scales + (int64_t)bh * p.cache_tokens * L::kScale;

  // The key that this lane's row x of a tile holds in the cache.
  auto cache_row = [&](int64_t key) {
    int64_t r = p.first_row + key;
    return r >= p.cache_tokens ? r - p.cache_tokens : r;
  };
  auto fetch = [&](int64_t j, int stage) {
    if (j < j1) {
      const int64_t key0 = first + j * kKeys;
      const uint32_t dst = ring_u + stage * L::bytes;
      constexpr int kPieces = L::kRow / 16;  // 16-byte pieces of a row
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int x = i * 32 + lane;
        const int r = x / kPieces, piece = x % kPieces;
        const bool ok = key0 + r < p.keys;
        const int64_t at =
            (ok ? cache_row(key0 + r) : 0) * L::kRow + piece * 16;
        copy_async<16>(dst + L::k + r * L::kRow + piece * 16, k_codes + at, ok);
        copy_async<16>(dst + L::v + v_offset<D>(r, piece * 16), v_codes + at,
                       ok);
      }
      const bool ok = key0 + lane < p.keys;
      const int64_t at = (ok ? cache_row(key0 + lane) : 0) * L::kScale;
      copy_async<L::kScale>(dst + L::ks + lane * L::kScale, k_scales + at, ok);
      copy_async<L::kScale>(dst + L::vs + lane * L::kScale, v_scales + at, ok);
    }
    copy_commit();
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) fetch(j0 + warp + s * W, s);

  // Q^T fragments: for group i, element pairs (e, e + 4) of words 4 i + c.
  uint32_t qf[NT][kGroups][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = (rb * NT + nt) * 8 + g;
    const int tok = row / p.group, head = hk * p.group + row % p.group;
    const uint16_t* q =
        p.q + (((int64_t)b * p.q_tokens + tok) * p.heads + head) * D;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (row < p.rows)
        w = *reinterpret_cast<const uint4*>(q + 32 * i + 8 * c);
      qf[nt][i][0] = __byte_perm(w.x, w.z, 0x5410);
      qf[nt][i][1] = __byte_perm(w.x, w.z, 0x7632);
      qf[nt][i][2] = __byte_perm(w.y, w.w, 0x5410);
      qf[nt][i][3] = __byte_perm(w.y, w.w, 0x7632);
    }
  }

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
  for (int64_t j = j0 + warp; j < j1; j += W) {
    copy_wait<kStages - 2>();
    __syncwarp();
    {
      int ahead = stage + kStages - 1;
      if (ahead >= kStages) ahead -= kStages;
      fetch(j + (int64_t)(kStages - 1) * W, ahead);
    }
    const uint8_t* t = ring + stage * L::bytes;
    if (++stage == kStages) stage = 0;

    // S^T: two blocks of 16 keys
    float s[NT][2][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][x][e] = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t w[2][kGroups], sc[2][kGroups];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = x * 16 + y * 8 + kr;
        if constexpr (D == 128) {
          const uint4 v = *reinterpret_cast<const uint4*>(t + L::k +
                                                          r * L::kRow + c * 16);
          w[y][0] = v.x, w[y][1] = v.y, w[y][2] = v.z, w[y][3] = v.w;
          const uint2 f =
              *reinterpret_cast<const uint2*>(t + L::ks + r * L::kScale);
          sc[y][0] = __byte_perm(f.x, f.x, 0x1010);
          sc[y][1] = __byte_perm(f.x, f.x, 0x3232);
          sc[y][2] = __byte_perm(f.y, f.y, 0x1010);
          sc[y][3] = __byte_perm(f.y, f.y, 0x3232);
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(t + L::k +
                                                          r * L::kRow + c * 8);
          w[y][0] = v.x, w[y][1] = v.y;
          const uint32_t f =
              *reinterpret_cast<const uint32_t*>(t + L::ks + r * L::kScale);
          sc[y][0] = __byte_perm(f, f, 0x1010);
          sc[y][1] = __byte_perm(f, f, 0x3232);
        }
      }
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const uint32_t o0 = scale_offset(sc[0][i]), o1 = scale_offset(sc[1][i]);
        uint32_t a[4];
        a[0] = expand<0>(w[0][i], sc[0][i], o0);
        a[1] = expand<0>(w[1][i], sc[1][i], o1);
        a[2] = expand<1>(w[0][i], sc[0][i], o0);
        a[3] = expand<1>(w[1][i], sc[1][i], o1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          mma(s[nt][x], a, qf[nt][i][0], qf[nt][i][1]);
        a[0] = expand<2>(w[0][i], sc[0][i], o0);
        a[1] = expand<2>(w[1][i], sc[1][i], o1);
        a[2] = expand<3>(w[0][i], sc[0][i], o0);
        a[3] = expand<3>(w[1][i], sc[1][i], o1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          mma(s[nt][x], a, qf[nt][i][2], qf[nt][i][3]);
      }
    }

    // Softmax over the tile's 32 keys; lane: keys x 16 + e/2 8 + kr of rows
    // 2 c + e % 2.
    const int64_t left = p.keys - first - j * kKeys;
    uint32_t pt[NT][2][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = s[nt][x][e] * p.scale_log2;
          if (left < kKeys && x * 16 + (e / 2) * 8 + kr >= left) v = -INFINITY;
          s[nt][x][e] = v;
          top[e % 2] = fmaxf(top[e % 2], v);
        }
#pragma unroll
      for (int y = 4; y < 32; y *= 2) {
        top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], y));
        top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], y));
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
          s[nt][x][e] = ex2(s[nt][x][e] - m[nt][e % 2]);
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
#define FASTVR_PV(J)                                              \
  {                                                               \
    const uint32_t a[4] = {                                       \
        expand<J>(a00, s0, o0), expand<J>(a01, s0, o0),           \
        expand<J>(a10, s1, o1), expand<J>(a11, s1, o1)};          \
    _Pragma("unroll") for (int nt = 0; nt < NT; ++nt)             \
        mma(o[nt][4 * i + J], a, pt[nt][x][0], pt[nt][x][1]);     \
  }
        FASTVR_PV(0) FASTVR_PV(1) FASTVR_PV(2) FASTVR_PV(3)
#undef FASTVR_PV
      }
    }
  }
  copy_wait<0>();
  __syncwarp();

  // Join the warps: each leaves m, l and O[row][d] (for its own m) in its
  // part of shared memory.
  float* so = reinterpret_cast<float*>(ring);
  constexpr int kPitch = D + 4;
  static_assert(kRows * kPitch * 4 <= kStages * L::bytes, "ring too small");
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float x = l[nt][q];
#pragma unroll
      for (int y = 4; y < 32; y *= 2) x += __shfl_xor_sync(0xffffffffu, x, y);
      const int row = nt * 8 + 2 * c + q;
      if (g == 0) {
        s_m[warp][row] = m[nt][q];
        s_l[warp][row] = x;
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

  const int unit = bh * p.row_blocks + rb;
  const int rows = min(kRows, p.rows - rb * kRows);
  float* part = p.partial +
                ((int64_t)unit * p.splits + split) * kRows * (D + 2);
  auto finish = [&](int row, int d, float acc, float sum, float top) {
    const int r = rb * kRows + row;
    const int tok = r / p.group, head = hk * p.group + r % p.group;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // no key: zeros
    p.out[(((int64_t)b * p.q_tokens + tok) * p.heads + head) * D + d] =
        __bfloat16_as_ushort(__float2bfloat16_rn(acc * inv));
    if (d == 0 && p.lse != nullptr)
      p.lse[((int64_t)b * p.heads + head) * p.q_tokens + tok] =
          sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
  };
  for (int x = threadIdx.x; x < rows * D; x += W * 32) {
    const int row = x / D, d = x % D;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, s_m[w][row]);
    float acc = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      // a warp without keys (m = -inf, l = 0) adds nothing
      const float mw = s_m[w][row];
      const float f = mw == -INFINITY && s_l[w][row] == 0.f ? 0.f : ex2(mw - top);
      const float* src =
          reinterpret_cast<const float*>(smem + w * kStages * L::bytes);
      acc = fmaf(f, src[row * kPitch + d], acc);
      sum = fmaf(f, s_l[w][row], sum);
    }
    if (p.splits == 1) {
      finish(row, d, acc, sum, top);
    } else {
      part[row * (D + 2) + d] = acc;
      if (d == 0) {
        part[row * (D + 2) + D] = top;
        part[row * (D + 2) + D + 1] = sum;
      }
    }
  }
  if (p.splits == 1) return;

  // The last CTA of the unit to arrive joins the key ranges, in their order.
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const int n = atomicAdd(p.tickets + unit, 1);
    s_last = n == p.splits - 1;
    if (s_last) p.tickets[unit] = 0;  // for the next call
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  const float* all = p.partial + (int64_t)unit * p.splits * kRows * (D + 2);
  for (int x = threadIdx.x; x < rows * D; x += W * 32) {
    const int row = x / D, d = x % D;
    float top = -INFINITY, acc = 0.f, sum = 0.f;
    for (int i = 0; i < p.splits; ++i) {
      const float* src = all + ((int64_t)i * kRows + row) * (D + 2);
      const float mi = __ldcg(src + D), li = __ldcg(src + D + 1);
      const float oi = __ldcg(src + d);
      if (mi == -INFINITY && li == 0.f) continue;  // no keys in this range
      const float mn = fmaxf(top, mi);
      const float f0 = top == -INFINITY ? 0.f : ex2(top - mn);
      const float f1 = ex2(mi - mn);
      acc = fmaf(oi, f1, acc * f0);
      sum = fmaf(li, f1, sum * f0);
      top = mn;
    }
    finish(row, d, acc, sum, top);
  }
}

constexpr int kWarps = 8;

template <int D, int NT, int kStages>
cudaError_t launch_v(Q4AttnParams p, int sms, cudaStream_t stream) {
  p.row_blocks = (p.rows + 8 * NT - 1) / (8 * NT);
  const int64_t units = (int64_t)p.batch_heads * p.row_blocks;
  // Cut the keys so that the CTAs fill the SMs: the number of splits with the
  // shortest time, counted in key tiles of the longest warp plus a fixed cost
  // of about 4 tiles per CTA.
  const int64_t tiles = (p.keys + kKeys - 1) / kKeys;
  const int64_t slots = sms;
  int64_t best = 1, best_cost = INT64_MAX;
  for (int64_t s = 1; s <= kQ4MaxSplits && units * s <= kQ4MaxParts; ++s) {
    if (s > 1 && (tiles + s - 1) / s < kWarps) break;
    const int64_t waves = (units * s + slots - 1) / slots;
    const int64_t per = (tiles + s * kWarps - 1) / (s * kWarps);
    const int64_t cost = waves * (per + 4);
    if (cost < best_cost) {
      best_cost = cost;
      best = s;
    }
  }
  p.splits = (int32_t)best;
  const int64_t grid = units * best;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  constexpr int smem = kWarps * kStages * Tile<D>::bytes;
  auto kernel = q4_attn_kernel<D, NT, kWarps, kStages>;
  const cudaError_t e = cudaFuncSetAttribute(
      kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(kWarps * 32), smem,
                    stream, p);
}

template <int D>
cudaError_t launch_d(const Q4AttnParams& p, int sms, cudaStream_t stream) {
  constexpr int kStages = D == 128 ? 4 : 8;
  if (p.rows <= 8) return launch_v<D, 1, kStages>(p, sms, stream);
  if (p.rows <= 16) return launch_v<D, 2, kStages>(p, sms, stream);
  return launch_v<D, 4, kStages>(p, sms, stream);
}

}  // namespace

cudaError_t launch_q4_attn(const Q4AttnParams& p, int sms,
                           cudaStream_t stream) {
  if (p.head_dim == 64) return launch_d<64>(p, sms, stream);
  if (p.head_dim == 128) return launch_d<128>(p, sms, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastvr
