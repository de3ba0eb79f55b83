// Cross attention of few query rows (single tokens): bound by reading the keys
// and values once, and by latency.
//
// The rows of a (batch entry, key head) are its tokens times the query heads that
// share the key head, in blocks of 16: one warp-level product has them as its
// rows.  A cluster of CTAs shares a block's keys, a CTA's eight warps take 16
// keys each in turn, straight from memory to registers, with running maxima and
// sums per warp; the warps' results are joined through shared memory, the CTAs'
// through the cluster's, so there is no scratch and one launch.  12 heads over 77
// keys take 4.1 us (latency), 16 streams of 32 heads over 8 and up to 512 keys 9.6
// (the longest prompt's CTA; 2.6 us of bytes).
//
// Both summed axes are permuted so that lanes read whole pieces of rows: for
// S = q k^T a lane (g = lane / 4, t = lane % 4) holds elements 8 t .. 8 t + 7 of
// every 32 of a row; for O = P v column g of block n is element g d / 8 + n of
// the head, so a lane reads d / 8 neighbouring elements of a value row.
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "attn_softmax.cuh"
#include "cross_attn.cuh"
#include "fastvr_internal.h"
#include "mma_sync.cuh"
#include "sm100_ptx.cuh"

namespace fastvr {
namespace {

constexpr int kWarps = 8;
constexpr int kKeys = 16;  // of a warp at a time

struct RowsParams {
  CrossArgs a;
  int32_t group, rows, blocks;  // of a (batch entry, key head)
  FastDiv by_blocks, by_heads, by_group;
  float scale_log2;
};

template <int D>
struct RowsShared {
  float o[kWarps][kCrossRows][D + 4];  // the CTA's sum lands in o[0]
  float m[kWarps][kCrossRows], l[kWarps][kCrossRows];
  float cta_m[kCrossRows], cta_l[kCrossRows];
};

__device__ __forceinline__ float load_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 1)
cross_rows_kernel(const __grid_constant__ RowsParams p) {
  using sm100::cluster_addr;
  extern __shared__ __align__(16) uint8_t smem[];
  RowsShared<D>& S = *reinterpret_cast<RowsShared<D>*>(smem);
  constexpr int kPieces = D / 32;  // 16-byte pieces of a row that a lane holds
  constexpr int kCols = D / 8;     // blocks of 8 output columns
  const CrossArgs& a = p.a;
  uint32_t ctas, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int g = lane / 4, t = lane % 4;
  const uint32_t unit = blockIdx.x / ctas;
  const uint32_t bh = fast_div(unit, p.by_blocks);
  const int row0 = (int)(unit - bh * p.blocks) * kCrossRows;
  const int b = (int)fast_div(bh, p.by_heads);
  const int hk = (int)(bh - (uint32_t)b * a.kv_heads);
  pdl_trigger();
  pdl_wait();
  const int len = cross_keys(a.kv_len, b, a.kv_tokens);

  // Rows g and g + 8 of the block.
  uint4 q[2][kPieces];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = row0 + g + 8 * i;
    const int tok = (int)fast_div(r, p.by_group);
    const int h = hk * p.group + r - tok * p.group;
#pragma unroll
    for (int c = 0; c < kPieces; ++c) {
      q[i][c] = make_uint4(0, 0, 0, 0);
      if (r < p.rows)
        q[i][c] = __ldg(reinterpret_cast<const uint4*>(
            a.q + (int64_t)b * a.q_str.batch + (int64_t)tok * a.q_str.token +
            (int64_t)h * a.q_str.head + 32 * c + 8 * t));
    }
  }
  const uint16_t* k = a.k + (int64_t)b * a.k_str.batch +
                      (int64_t)hk * a.k_str.head + 8 * t;
  const uint16_t* v = a.v + (int64_t)b * a.v_str.batch +
                      (int64_t)hk * a.v_str.head + g * kCols;
  float o[kCols][4];
#pragma unroll
  for (int n = 0; n < kCols; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  const int step = (int)ctas * kWarps * kKeys;
  for (int j = ((int)rank * kWarps + warp) * kKeys; j < len; j += step) {
    // keys j + g and j + 8 + g; value rows j + 2 t, + 1, + 8, + 9
    uint4 kk[2][kPieces];
    uint32_t vv[4][kCols / 2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = j + 8 * i + g;
#pragma unroll
      for (int c = 0; c < kPieces; ++c) {
        kk[i][c] = make_uint4(0, 0, 0, 0);
        if (key < len)
          kk[i][c] = __ldg(reinterpret_cast<const uint4*>(
              k + (int64_t)key * a.k_str.token + 32 * c));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = j + 2 * t + (i & 1) + 8 * (i >> 1);
#pragma unroll
      for (int c = 0; c < kCols / 8; ++c) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (key < len)
          x = __ldg(reinterpret_cast<const uint4*>(
              v + (int64_t)key * a.v_str.token + 8 * c));
        vv[i][4 * c] = x.x;
        vv[i][4 * c + 1] = x.y;
        vv[i][4 * c + 2] = x.z;
        vv[i][4 * c + 3] = x.w;
      }
    }
    float s[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = 0.f;
#pragma unroll
      for (int c = 0; c < kPieces; ++c) {
        mma_16x8x16(s[i], q[0][c].x, q[1][c].x, q[0][c].y, q[1][c].y,
                    kk[i][c].x, kk[i][c].y);
        mma_16x8x16(s[i], q[0][c].z, q[1][c].z, q[0][c].w, q[1][c].w,
                    kk[i][c].z, kk[i][c].w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[i][e] = j + 8 * i + 2 * t + (e & 1) < len ? s[i][e] * p.scale_log2
                                                    : -INFINITY;
    }
    float alpha[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]),
                      fmaxf(s[1][2 * r], s[1][2 * r + 1]));
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
      const float top = fmaxf(m[r], x);
      // a row whose scores are all -infinity so far exponentiates against 0
      const float ref = top == -INFINITY ? 0.f : top;
      alpha[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - ref);
      m[r] = top;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[i][2 * r + e] = ex2(s[i][2 * r + e] - ref);
          sum += s[i][2 * r + e];
        }
      l[r] = l[r] * alpha[r] + sum;
    }
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      o[n][0] *= alpha[0];
      o[n][1] *= alpha[0];
      o[n][2] *= alpha[1];
      o[n][3] *= alpha[1];
    }
    // P in bfloat16, V's type; the sums above took it unrounded
    const uint32_t a0 = pack_bf16(s[0][0], s[0][1]),
                   a1 = pack_bf16(s[0][2], s[0][3]),
                   a2 = pack_bf16(s[1][0], s[1][1]),
                   a3 = pack_bf16(s[1][2], s[1][3]);
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      const uint32_t pick = n & 1 ? 0x7632u : 0x5410u;
      mma_16x8x16(o[n], a0, a1, a2, a3,
                  __byte_perm(vv[0][n / 2], vv[1][n / 2], pick),
                  __byte_perm(vv[2][n / 2], vv[3][n / 2], pick));
    }
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(~0u, l[r], 1);
    l[r] += __shfl_xor_sync(~0u, l[r], 2);
    if (t == 0) {
      S.m[warp][g + 8 * r] = m[r];
      S.l[warp][g + 8 * r] = l[r];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int n = 0; n < kCols; n += 4)
        *reinterpret_cast<float4*>(
            &S.o[warp][g + 8 * r][(2 * t + e) * kCols + n]) =
            make_float4(o[n][2 * r + e], o[n + 1][2 * r + e],
                        o[n + 2][2 * r + e], o[n + 3][2 * r + e]);
  }
  __syncthreads();
  // The CTA's rows: 16 lanes to a row, D / 16 elements each.
  {
    const int r = threadIdx.x / 16, x0 = threadIdx.x % 16 * (D / 16);
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, S.m[w][r]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, acc[D / 16];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) acc[x] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2(S.m[w][r] - ref);
      sum += f * S.l[w][r];
#pragma unroll
      for (int x = 0; x < D / 16; x += 4) {
        const float4 v4 = *reinterpret_cast<const float4*>(&S.o[w][r][x0 + x]);
        acc[x] += f * v4.x;
        acc[x + 1] += f * v4.y;
        acc[x + 2] += f * v4.z;
        acc[x + 3] += f * v4.w;
      }
    }
    // nothing else reads these places of o[0]
#pragma unroll
    for (int x = 0; x < D / 16; x += 4)
      *reinterpret_cast<float4*>(&S.o[0][r][x0 + x]) =
          make_float4(acc[x], acc[x + 1], acc[x + 2], acc[x + 3]);
    if (x0 == 0) {
      S.cta_m[r] = top;
      S.cta_l[r] = sum;
    }
  }
  if (ctas > 1)
    sm100::cluster_sync();
  else
    __syncthreads();
  // Pieces of 8 elements of the rows, dealt to the cluster's CTAs.
  const int pieces = min(kCrossRows, p.rows - row0) * (D / 8);
  for (int i = (int)rank * (kWarps * 32) + threadIdx.x; i < pieces;
       i += (int)ctas * kWarps * 32) {
    const int rr = i / (D / 8), x0 = i % (D / 8) * 8;
    float top = -INFINITY, sum = 0.f, acc[8] = {};
    for (uint32_t c = 0; c < ctas; ++c)
      top = fmaxf(top, load_cluster(cluster_addr(&S.cta_m[rr], c)));
    const float ref = top == -INFINITY ? 0.f : top;
    for (uint32_t c = 0; c < ctas; ++c) {
      const float f = ex2(load_cluster(cluster_addr(&S.cta_m[rr], c)) - ref);
      sum += f * load_cluster(cluster_addr(&S.cta_l[rr], c));
      const uint32_t from = cluster_addr(&S.o[0][rr][x0], c);
#pragma unroll
      for (int x = 0; x < 8; ++x) acc[x] += f * load_cluster(from + 4 * x);
    }
    const float inv = len == 0 ? 0.f : 1.f / sum;
    const int r = row0 + rr;
    const int tok = (int)fast_div(r, p.by_group);
    const int h = hk * p.group + r - tok * p.group;
    *reinterpret_cast<uint4*>(a.o + (int64_t)b * a.o_str.batch +
                              (int64_t)tok * a.o_str.token +
                              (int64_t)h * a.o_str.head + x0) =
        make_uint4(pack_bf16(acc[0] * inv, acc[1] * inv),
                   pack_bf16(acc[2] * inv, acc[3] * inv),
                   pack_bf16(acc[4] * inv, acc[5] * inv),
                   pack_bf16(acc[6] * inv, acc[7] * inv));
    if (a.lse != nullptr && x0 == 0)
      a.lse[((int64_t)b * a.heads + h) * a.q_tokens + tok] =
          len == 0 ? -INFINITY
                   : (top + __log2f(sum)) * 0.6931471805599453f;
  }
  if (ctas > 1) sm100::cluster_sync();  // nobody leaves while it is read
}

template <int D>
cudaError_t launch_d(const CrossArgs& a, cudaStream_t stream) {
  RowsParams p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  p.group = a.heads / a.kv_heads;
  p.rows = a.q_tokens * p.group;
  p.blocks = (p.rows + kCrossRows - 1) / kCrossRows;
  p.by_blocks = make_div((uint32_t)p.blocks);
  p.by_heads = make_div((uint32_t)a.kv_heads);
  p.by_group = make_div((uint32_t)p.group);
  p.scale_log2 = a.scale * 1.4426950408889634f;
  // As many CTAs to a block's keys as keep every SM at one CTA, and each warp at
  // 16 keys or more.
  const int units = a.batch * a.kv_heads * p.blocks;
  int ctas = 1;
  while (ctas < 8 && 2 * ctas * units <= a.sms &&
         ctas * kWarps * kKeys < a.kv_tokens)
    ctas *= 2;
  const int smem = (int)sizeof(RowsShared<D>);
  const cudaError_t e = allow_smem<cross_rows_kernel<D>>(smem, a.device);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * ctas));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ctas;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, cross_rows_kernel<D>, p);
}

}  // namespace

cudaError_t launch_cross_rows(const CrossArgs& a, cudaStream_t stream) {
  return a.head_dim == 64 ? launch_d<64>(a, stream)
                          : launch_d<128>(a, stream);
}

}  // namespace fastvr
