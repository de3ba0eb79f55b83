// Between two blocks: r = a x + gate o post(y), h = pre(r) o (1 + scale) +
// shift, in one pass over memory.
//
// Bound by memory: x and y are read once, r and h written once (8 bytes per
// element in bfloat16).  A row lives in the registers of its threads (one
// warp up to dim 1536, so that its sums need no shared memory), which makes
// mean and variance two exact passes at no cost in traffic.  The modulation
// vectors are shared by all tokens of a group and come from L1/L2.
#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

constexpr int kThreads = 128;  // of a CTA whose rows take one warp each

template <typename TR, typename TY, int TPR, int NV>
__global__ void __launch_bounds__(TPR > kThreads ? TPR : kThreads)
norm_fwd_kernel(const __grid_constant__ NormFwdParams p) {
  __shared__ float smem[2 * (TPR / 32)];
  constexpr int kRows = TPR == 32 ? kThreads / 32 : 1;
  const int64_t row =
      (int64_t)blockIdx.x * kRows + (kRows > 1 ? threadIdx.x / TPR : 0);
  const int lane = threadIdx.x % TPR;
  pdl_trigger();
  pdl_wait();
  if (row >= p.rows) return;  // a whole warp (TPR = 32), or never
  const int64_t base = row * p.dim;
  const int64_t mod = row / p.group_tokens * p.dim;
  const float inv_dim = 1.f / (float)p.dim;

  Raw8<TR> xr[NV];
  Raw8<TY> yr[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    if (c < p.dim) {
      xr[i].load(p.x, base + c);
      if (p.y != nullptr) yr[i].load(p.y, base + c);
    }
  }
  float r[NV][8];
  float mu = 0.f, rho = 1.f;
  if (p.y != nullptr) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if ((i * TPR + lane) * 8 < p.dim) {
        yr[i].widen(r[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[i][e] = 0.f;
      }
    }
    if (p.post != kNormNone) {
      if (p.post == kNormLayer) {
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) s[0] += sum8(r[i]);
        row_sum<TPR>(s, smem);
        mu = s[0] * inv_dim;
      }
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((i * TPR + lane) * 8 < p.dim)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = r[i][e] - mu;
            s[0] = fmaf(d, d, s[0]);
          }
      row_sum<TPR>(s, smem);
      rho = rsqrtf(s[0] * inv_dim + p.eps);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    if (c < p.dim) {
      float x[8];
      xr[i].widen(x);
      if (p.y != nullptr) {
        float g[8], w[8];
        load8_or(p.gate, mod + c, 1.f, g);
        load8_or(p.post == kNormNone ? nullptr : p.post_weight, c, 1.f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = (r[i][e] - mu) * rho * w[e];
          r[i][e] = fmaf(g[e], u, p.residual_scale * x[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[i][e] = p.residual_scale * x[e];
      }
      if (p.r != nullptr) store8(static_cast<TR*>(p.r), base + c, r[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[i][e] = 0.f;
    }
  }
  if (p.h == nullptr) return;

  mu = 0.f;
  if (p.pre == kNormLayer) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) s[0] += sum8(r[i]);
    row_sum<TPR>(s, smem);
    mu = s[0] * inv_dim;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if ((i * TPR + lane) * 8 < p.dim)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = r[i][e] - mu;
        s[0] = fmaf(d, d, s[0]);
      }
  row_sum<TPR>(s, smem);
  rho = rsqrtf(s[0] * inv_dim + p.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    if (c < p.dim) {
      float sc[8], sh[8], w[8];
      load8_or(p.scale, mod + c, 0.f, sc);
      load8_or(p.shift, mod + c, 0.f, sh);
      load8_or(p.pre_weight, c, 1.f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        r[i][e] = fmaf((r[i][e] - mu) * rho * w[e], 1.f + sc[e], sh[e]);
      store8(static_cast<TY*>(p.h), base + c, r[i]);
    }
  }
}

template <typename TR, typename TY, int TPR, int NV>
cudaError_t launch_v(const NormFwdParams& p, cudaStream_t stream) {
  constexpr int kRows = TPR == 32 ? kThreads / 32 : 1;
  const int64_t grid = (p.rows + kRows - 1) / kRows;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_pdl(norm_fwd_kernel<TR, TY, TPR, NV>, dim3((unsigned)grid),
                    dim3(TPR == 32 ? kThreads : TPR), 0, stream, p);
}

// Threads per row and vectors of 8 per thread: the smallest that hold dim.
template <typename TR, typename TY>
cudaError_t launch_t(const NormFwdParams& p, cudaStream_t stream) {
  if (p.dim <= 256) return launch_v<TR, TY, 32, 1>(p, stream);
  if (p.dim <= 512) return launch_v<TR, TY, 32, 2>(p, stream);
  if (p.dim <= 1024) return launch_v<TR, TY, 32, 4>(p, stream);
  if (p.dim <= 1536) return launch_v<TR, TY, 32, 6>(p, stream);
  if (p.dim <= 2048) return launch_v<TR, TY, 128, 2>(p, stream);
  if (p.dim <= 4096) return launch_v<TR, TY, 128, 4>(p, stream);
  return launch_v<TR, TY, 256, 4>(p, stream);
}

}  // namespace

cudaError_t launch_norm_fwd(const NormFwdParams& p, bool res_f32,
                            bool block_f32, cudaStream_t stream) {
  using B = __nv_bfloat16;
  if (res_f32)
    return block_f32 ? launch_t<float, float>(p, stream)
                     : launch_t<float, B>(p, stream);
  return block_f32 ? launch_t<B, float>(p, stream) : launch_t<B, B>(p, stream);
}

}  // namespace fastvr
