// Gated feed-forward of few tokens, h = act(x Wg^T) o (x Wu^T): bound by reading
// the weights once.
//
// A CTA forms 8 or 16 columns of h for all tokens.  One warp-level product has 8 rows
// of Wg over the same 8 of Wu as its 16 rows and 8 tokens as its columns, so a
// lane ends up with g and u of the same column and token.  The eight warps take
// 128-byte pieces of the rows in turn (a row's pieces of one pass are 1 KB) and
// their sums are added through shared memory in order.  One token of 1536 to 4096
// takes 6.8 us (25 MB of weights: 3.8 us), 16 tokens 8.7: every CTA reads all of x.
#include <cuda_bf16.h>
#include <math.h>

#include "ffn_act.cuh"
#include "fastvr_internal.h"
#include "mma_sync.cuh"

namespace fastvr {
namespace {

constexpr int kWarps = 8;
constexpr int kPiece = 64;  // elements of a row that four lanes read

// kTok: blocks of 8 tokens; kCols: blocks of 8 columns of a CTA.  With more tokens
// a CTA takes two, or it would read more of x than of the weights (24 tokens of 1536
// to 4096 10.4 us with one).  Three CTAs to an SM, for which the compiler spills a
// little from 17 tokens on: 2048 to 5632 is 352 CTAs, 17.4 us with two to an SM.
template <int kTok, int kCols, int kAct>
__global__ void __launch_bounds__(kWarps * 32, 3)
rows_kernel(const __grid_constant__ FfnArgs a) {
  __shared__ float part[kWarps][kCols * kTok][32][4];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int g = lane / 4, t = lane % 4;
  const int f0 = blockIdx.x * 8 * kCols;
  float c[kCols][kTok][4];
#pragma unroll
  for (int f = 0; f < kCols; ++f)
#pragma unroll
    for (int n = 0; n < kTok; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) c[f][n][e] = 0.f;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  // eight loads of weights in flight: two pieces of a row, or one of two
  constexpr int kLoads = 4 / kCols;
  for (int k0 = warp * kPiece; k0 < a.dim;
       k0 += kLoads / 2 * kWarps * kPiece) {
    uint4 vg[kCols][kLoads], vu[kCols][kLoads];
#pragma unroll
    for (int f = 0; f < kCols; ++f) {
      const int row = f0 + 8 * f + g;
      const uint16_t* wg = a.w_gate + (int64_t)row * a.dim;
      const uint16_t* wu = a.w_up + (int64_t)row * a.dim;
#pragma unroll
      for (int s = 0; s < kLoads; ++s) {
        const int k = k0 + (s / 2) * kWarps * kPiece + (s % 2) * 32 + 8 * t;
        vg[f][s] = vu[f][s] = zero;
        if (k < a.dim && row < a.hidden) {
          vg[f][s] = load_once(wg + k);
          vu[f][s] = load_once(wu + k);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < kTok; ++n) {
      const bool in = n * 8 + g < a.tokens;
      const uint16_t* x = a.x + (int64_t)(n * 8 + g) * a.x_row;
#pragma unroll
      for (int s = 0; s < kLoads; ++s) {
        const int k = k0 + (s / 2) * kWarps * kPiece + (s % 2) * 32 + 8 * t;
        uint4 v = zero;
        if (in && k < a.dim) v = __ldg(reinterpret_cast<const uint4*>(x + k));
#pragma unroll
        for (int f = 0; f < kCols; ++f) {
          mma_16x8x16(c[f][n], vg[f][s].x, vu[f][s].x, vg[f][s].y, vu[f][s].y,
                      v.x, v.y);
          mma_16x8x16(c[f][n], vg[f][s].z, vu[f][s].z, vg[f][s].w, vu[f][s].w,
                      v.z, v.w);
        }
      }
    }
  }
#pragma unroll
  for (int f = 0; f < kCols; ++f)
#pragma unroll
    for (int n = 0; n < kTok; ++n)
      *reinterpret_cast<float4*>(part[warp][f * kTok + n][lane]) =
          make_float4(c[f][n][0], c[f][n][1], c[f][n][2], c[f][n][3]);
  __syncthreads();
  // Warp i joins block i: lane (g, t) holds g of column 8 f + g for tokens 2t and
  // 2t + 1 of block n, then u.
  for (int i = warp; i < kCols * kTok; i += kWarps) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(part[w][i][lane]);
      s[0] += v.x;
      s[1] += v.y;
      s[2] += v.z;
      s[3] += v.w;
    }
    const int col = f0 + i / kTok * 8 + g;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t tok = i % kTok * 8 + 2 * t + e;
      if (tok >= a.tokens || col >= a.hidden) continue;
      const int64_t at = tok * a.hidden + col;
      if (a.g != nullptr) {  // in bfloat16, as gated_ffn.cu keeps them
        a.g[at] = __bfloat16_as_ushort(__float2bfloat16_rn(s[e]));
        a.u[at] = __bfloat16_as_ushort(__float2bfloat16_rn(s[2 + e]));
      }
      a.h[at] = __bfloat16_as_ushort(
          __float2bfloat16_rn(activation<kAct>(s[e]) * s[2 + e]));
    }
  }
}

template <int kTok, int kCols>
cudaError_t launch_act(const FfnArgs& a, cudaStream_t stream) {
  const auto kernel = a.act == kActSilu   ? rows_kernel<kTok, kCols, kActSilu>
                      : a.act == kActGelu ? rows_kernel<kTok, kCols, kActGelu>
                                          : rows_kernel<kTok, kCols, kActGeluTanh>;
  return launch_pdl(kernel, dim3((a.hidden + 8 * kCols - 1) / (8 * kCols)),
                    dim3(kWarps * 32), 0, stream, a);
}

}  // namespace

cudaError_t launch_ffn_rows(const FfnArgs& a, cudaStream_t stream) {
  static_assert(kFfnMaxRows == 32, "a kernel for every number of blocks");
  switch ((a.tokens + 7) / 8) {
    case 1:
      return launch_act<1, 1>(a, stream);
    case 2:
      return launch_act<2, 2>(a, stream);
    case 3:
      return launch_act<3, 2>(a, stream);
    default:
      return launch_act<4, 2>(a, stream);
  }
}

}  // namespace fastvr
