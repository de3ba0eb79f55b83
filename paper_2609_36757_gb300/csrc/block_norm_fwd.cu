// Between two blocks: r = a x + gate o post(y), h = pre(r) o (1 + scale) +
// shift, in one pass over memory.
//
// Bound by memory: x and y are read once, r and h written once (8 bytes per
// element in bfloat16).  A thread owns 8 columns for all the rows that its CTA
// takes, so the modulation vectors of a group are read once and stay in its
// registers (with a warp to a row they were read again for every row, which
// kept L1 busier than memory), and two rows go through the sums together,
// the next two on their way.
#include <algorithm>

#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

template <typename TR, typename TY, int TPR, int kMinCtas>
__global__ void __launch_bounds__(Shape<TPR>::kThreads, kMinCtas)
norm_fwd_kernel(const __grid_constant__ NormFwdParams p) {
  using S = Shape<TPR>;
  // rows of a pass: two, where a thread has the registers for them
  constexpr int R = TPR > 512 ? 1 : 2;
  __shared__ float4 s_y[S::kWarps], s_r[S::kWarps];
  pdl_trigger();
  const Cols k = make_cols<TPR>(p.dim);
  const int slot = S::kRows > 1 ? threadIdx.x / TPR : 0;
  const int r0 = (int)((int64_t)blockIdx.x * p.rows / gridDim.x);
  const int r1 = (int)((int64_t)(blockIdx.x + 1) * p.rows / gridDim.x);
  const bool has_y = p.y != nullptr, has_h = p.h != nullptr;
  const bool post = has_y && p.post != kNormNone;
  pdl_wait();

  // Rows rb + slot and rb + kRows + slot of a pass.
  Raw8<TR> xr[R];
  Raw8<TY> yr[R];
  auto fetch = [&](int rb) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = rb + i * S::kRows + slot;
      if (k.on && row < r1) {
        const int64_t at = (int64_t)row * p.dim + k.c;
        xr[i].load(p.x, at);
        if (has_y) yr[i].load(p.y, at);
      }
    }
  };
  // gate o post_weight, and (1 + scale) o pre_weight and shift, of the group
  // last asked for.
  float gp[8], sw[8], sh[8];
  uint32_t group_y = ~0u, group_h = ~0u;

  fetch(r0);
  // every thread makes every pass (barriers and shuffles inside)
  for (int rb = r0; rb < r1; rb += R * S::kRows) {
    // a pass with one exchange only: its part is not written again before
    // every thread has read it
    if (S::kMany && post != has_h) __syncthreads();
    float x[R][8], y[R][8];
    bool on[R];
    uint32_t group[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = rb + i * S::kRows + slot;
      on[i] = k.on && row < r1;
      group[i] = (uint32_t)row / (uint32_t)p.group_tokens;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.f;
      if (on[i]) {
        xr[i].widen(x[i]);
        if (has_y) yr[i].widen(y[i]);
      }
    }
    fetch(rb + R * S::kRows);

    Stats st = {0.f, 0.f, 0.f, 0.f};
    float rho[2] = {1.f, 1.f};
    if (post) {
      const bool mean = p.post == kNormLayer;
      st = row_stats<TPR>(y[0], y[R - 1], mean, mean, k, s_y);
      rho[0] = rsqrtf(st.sq_a * k.inv_dim + p.eps);
      rho[1] = rsqrtf(st.sq_b * k.inv_dim + p.eps);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float mu = i ? st.mu_b : st.mu_a;
      if (on[i]) {
        if (has_y && group[i] != group_y) {
          float w[8];
          group_y = group[i];
          load8_or(p.gate, (int64_t)group_y * p.dim + k.c, 1.f, gp);
          load8_or(post ? p.post_weight : nullptr, k.c, 1.f, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) gp[e] *= w[e];
        }
        if (has_y) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[i][e] = fmaf((y[i][e] - mu) * rho[i], gp[e],
                           p.residual_scale * x[i][e]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][e] *= p.residual_scale;
        }
        if (p.r != nullptr)
          store8(static_cast<TR*>(p.r),
                 (int64_t)(rb + i * S::kRows + slot) * p.dim + k.c, x[i]);
      }
    }
    if (!has_h) continue;
    const bool mean = p.pre == kNormLayer;
    st = row_stats<TPR>(x[0], x[R - 1], mean, mean, k, s_r);
    rho[0] = rsqrtf(st.sq_a * k.inv_dim + p.eps);
    rho[1] = rsqrtf(st.sq_b * k.inv_dim + p.eps);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float mu = i ? st.mu_b : st.mu_a;
      if (on[i]) {
        if (group[i] != group_h) {
          float w[8];
          group_h = group[i];
          load8_or(p.scale, (int64_t)group_h * p.dim + k.c, 0.f, sw);
          load8_or(p.shift, (int64_t)group_h * p.dim + k.c, 0.f, sh);
          load8_or(p.pre_weight, k.c, 1.f, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) sw[e] = (1.f + sw[e]) * w[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[i][e] = fmaf((x[i][e] - mu) * rho[i], sw[e], sh[e]);
        store8(static_cast<TY*>(p.h),
               (int64_t)(rb + i * S::kRows + slot) * p.dim + k.c, x[i]);
      }
    }
  }
}

template <typename TR, typename TY, int TPR, int kMinCtas>
cudaError_t launch_v(const NormFwdParams& p, int sms, cudaStream_t stream) {
  using S = Shape<TPR>;
  // One wave of CTAs, each with an equal share of the rows; with few rows
  // each takes a pass of its own.
  const int64_t passes = (p.rows + S::kRows - 1) / S::kRows;
  const int64_t grid = std::min<int64_t>((int64_t)sms * kMinCtas, passes);
  return launch_pdl(norm_fwd_kernel<TR, TY, TPR, kMinCtas>,
                    dim3((unsigned)grid),
                    dim3(S::kMany ? row_threads(p.dim) : S::kThreads), 0,
                    stream, p);
}

template <typename TR, typename TY>
cudaError_t launch_t(const NormFwdParams& p, int sms, cudaStream_t stream) {
  const int n = row_threads(p.dim);
  if (n == 8) return launch_v<TR, TY, 8, 4>(p, sms, stream);
  if (n == 16) return launch_v<TR, TY, 16, 4>(p, sms, stream);
  if (n == 32) return launch_v<TR, TY, 32, 4>(p, sms, stream);
  if (n <= 64) return launch_v<TR, TY, 64, 8>(p, sms, stream);
  if (n <= 128) return launch_v<TR, TY, 128, 4>(p, sms, stream);
  if (n <= 192) return launch_v<TR, TY, 192, 3>(p, sms, stream);
  if (n <= 256) return launch_v<TR, TY, 256, 2>(p, sms, stream);
  if (n <= 512) return launch_v<TR, TY, 512, 1>(p, sms, stream);
  return launch_v<TR, TY, 1024, 1>(p, sms, stream);
}

}  // namespace

cudaError_t launch_norm_fwd(const NormFwdParams& p, bool res_f32,
                            bool block_f32, int sms, cudaStream_t stream) {
  using B = __nv_bfloat16;
  if (res_f32)
    return block_f32 ? launch_t<float, float>(p, sms, stream)
                     : launch_t<float, B>(p, sms, stream);
  return block_f32 ? launch_t<B, float>(p, sms, stream)
                   : launch_t<B, B>(p, sms, stream);
}

}  // namespace fastvr
