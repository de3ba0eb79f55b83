// Gated feed-forward: h = act(x Wg^T) o (x Wu^T) and its gradients, as 64 x 64
// tiles in float32.
#include <cuda_bf16.h>
#include <math.h>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

// act(g) and its derivative in float32.
__device__ __forceinline__ float activation(float g, int act, float* slope) {
  if (act == kActSilu) {
    const float s = 1.f / (1.f + expf(-g));
    *slope = s * (1.f + g * (1.f - s));
    return g * s;
  }
  if (act == kActGelu) {
    const float c = 0.5f * (1.f + erff(g * 0.70710678f));
    *slope = c + g * 0.39894228f * expf(-0.5f * g * g);
    return g * c;
  }
  const float t = tanhf(0.79788456f * (g + 0.044715f * g * g * g));
  *slope = 0.5f * (1.f + t) + 0.5f * g * (1.f - t * t) * 0.79788456f *
                                  (1.f + 3.f * 0.044715f * g * g);
  return 0.5f * g * (1.f + t);
}

// c[m, n] = sum_k a[m, k] b[n, k] over two operand pairs one after the other
// (join) or side by side (h = act(c0) o c1); element strides for both axes.
struct Mat {
  const uint16_t* p;
  int64_t row, k;
};
struct Product {
  Mat a[2], b[2];
  int m, n, k, act;
  bool gated;
  uint16_t *c, *g, *u;  // [m, n]
};

__global__ void __launch_bounds__(256) product_kernel(Product p) {
  __shared__ float sa[16][65], sb[16][65];
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[2][4][4] = {};
  for (int pass = 0; pass < 2 && p.a[pass].p; ++pass)
    for (int k0 = 0; k0 < p.k; k0 += 16) {
      for (int i = threadIdx.x; i < 1024; i += 256) {
        const int r = i / 16, k = i % 16;
        const bool in = k0 + k < p.k;
        sa[k][r] = in && m0 + r < p.m
                       ? bf16_lo(p.a[pass].p[(m0 + r) * p.a[pass].row +
                                             (k0 + k) * p.a[pass].k])
                       : 0.f;
        sb[k][r] = in && n0 + r < p.n
                       ? bf16_lo(p.b[pass].p[(n0 + r) * p.b[pass].row +
                                             (k0 + k) * p.b[pass].k])
                       : 0.f;
      }
      __syncthreads();
      for (int k = 0; k < 16; ++k)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j) {
            const float t = sa[k][ty + 16 * i] * sb[k][tx + 16 * j];
            if (p.gated && pass)
              acc[1][i][j] += t;
            else
              acc[0][i][j] += t;
          }
      __syncthreads();
    }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= p.m || n >= p.n) continue;
      const int64_t x = (int64_t)m * p.n + n;
      float v = acc[0][i][j], slope;
      if (p.gated) {
        if (p.g) {
          p.g[x] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
          p.u[x] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[1][i][j]));
        }
        v = activation(v, p.act, &slope) * acc[1][i][j];
      }
      p.c[x] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
    }
}

__global__ void __launch_bounds__(256) slope_kernel(FfnBwdArgs a) {
  const int64_t n = (int64_t)a.f.tokens * a.f.hidden;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * 256) {
    float slope;
    const float g = bf16_lo(a.f.g[i]), u = bf16_lo(a.f.u[i]),
                d = bf16_lo(a.dh[i]);
    const float y = activation(g, a.f.act, &slope);
    a.dg[i] = __bfloat16_as_ushort(__float2bfloat16_rn(d * u * slope));
    a.du[i] = __bfloat16_as_ushort(__float2bfloat16_rn(d * y));
  }
}

cudaError_t launch_product(const Product& p, cudaStream_t stream) {
  const dim3 grid((p.n + 63) / 64, (p.m + 63) / 64);
  product_kernel<<<grid, 256, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_ffn_fwd(const FfnArgs& a, cudaStream_t stream) {
  Product p = {};
  p.a[0] = p.a[1] = {a.x, a.x_row, 1};
  p.b[0] = {a.w_gate, a.dim, 1};
  p.b[1] = {a.w_up, a.dim, 1};
  p.m = a.tokens;
  p.n = a.hidden;
  p.k = a.dim;
  p.act = a.act;
  p.gated = true;
  p.c = a.h;
  p.g = a.g;
  p.u = a.u;
  return launch_product(p, stream);
}

cudaError_t launch_ffn_bwd(const FfnBwdArgs& a, cudaStream_t stream) {
  slope_kernel<<<a.f.sms * 8, 256, 0, stream>>>(a);
  Product p = {};
  const int64_t F = a.f.hidden, D = a.f.dim;
  p.a[0] = {a.dg, F, 1};
  p.a[1] = {a.du, F, 1};
  p.b[0] = {a.f.w_gate, 1, D};
  p.b[1] = {a.f.w_up, 1, D};
  p.m = a.f.tokens;
  p.n = a.f.dim;
  p.k = a.f.hidden;
  p.c = a.dx;
  cudaError_t e = launch_product(p, stream);
  for (int i = 0; e == cudaSuccess && a.dw_gate && i < 2; ++i) {
    Product w = {};
    w.a[0] = {i ? a.du : a.dg, 1, F};
    w.b[0] = {a.f.x, 1, a.f.x_row};
    w.m = a.f.hidden;
    w.n = a.f.dim;
    w.k = a.f.tokens;
    w.c = i ? a.dw_up : a.dw_gate;
    e = launch_product(w, stream);
  }
  return e;
}

}  // namespace fastvr
