// Between two blocks: r = a x + gate o post(y), h = pre(r) o (1 + scale) +
// shift, in one pass over memory.
//
// Bound by memory: x and y are read once, r and h written once (8 bytes per
// element in bfloat16).  A thread owns the same columns of all the rows that
// its CTA takes, so the modulation vectors of a group are read and combined once
// (with a warp to a row they were read again for every row, which kept L1
// busier than memory) and kept in shared memory, and the next row is on its way
// while one goes through its sums.  What sets the time is the latency of a
// row's exchanges, so as many CTAs as fit without spilling share an SM: 37.9 us
// (5.3 TB/s) for 16320 rows of 1536 in bfloat16.
#include <algorithm>

#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

// R rows to a pass (of each row slot).
template <typename TR, typename TY, int TPR, int NV, int R, bool kAhead,
          int kMinCtas>
__global__ void __launch_bounds__(Shape<TPR>::kThreads, kMinCtas)
norm_fwd_kernel(const __grid_constant__ NormFwdParams p) {
  using S = Shape<TPR>;
  __shared__ float4 s_y[S::kWarps], s_r[S::kWarps];
  __shared__ float s_n[S::kWarps];
  extern __shared__ float4 dyn[];
  const Private mods = {dyn};
  pdl_trigger();
  const Cols<TPR, NV> k(p.dim, s_n);
  const int slot = S::kRows > 1 ? threadIdx.x / TPR : 0;
  const int r0 = (int)((int64_t)blockIdx.x * p.rows / gridDim.x);
  const int r1 = (int)((int64_t)(blockIdx.x + 1) * p.rows / gridDim.x);
  const bool has_y = p.y != nullptr, has_h = p.h != nullptr;
  const bool post = has_y && p.post != kNormNone;
  pdl_wait();

  // Rows rb + slot and rb + kRows + slot of a pass.
  Raw8<TR> xr[R][NV];
  Raw8<TY> yr[R][NV];
  auto fetch = [&](int rb) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = rb + i * S::kRows + slot;
      if (row < r1)
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (k.on(j)) {
            const int64_t at = (int64_t)row * p.dim + k.at(j);
            xr[i][j].load(p.x, at);
            if (has_y) yr[i][j].load(p.y, at);
          }
    }
  };
  // mods: gate o post_weight (j), (1 + scale) o pre_weight (NV + j) and shift
  // (2 NV + j) of the group last asked for.
  uint32_t group_y = ~0u, group_h = ~0u;

  if (kAhead) fetch(r0);
  // every thread makes every pass (barriers and shuffles inside)
  for (int rb = r0; rb < r1; rb += R * S::kRows) {
    // a pass with one exchange only: its part is not written again before
    // every thread has read it
    if (S::kMany && post != has_h) __syncthreads();
    if (!kAhead) fetch(rb);
    F8 x[R][NV], y[R][NV];
    bool on[R];
    uint32_t group[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = rb + i * S::kRows + slot;
      on[i] = row < r1;
      group[i] = fast_div(row, p.by_group_tokens);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        x[i][j] = on[i] && k.on(j) ? xr[i][j].widen() : splat(0.f);
        y[i][j] = on[i] && k.on(j) && has_y ? yr[i][j].widen() : splat(0.f);
      }
    }
    if (kAhead) fetch(rb + R * S::kRows);

    if (post) {
      const bool mean = p.post == kNormLayer;
      const Stats st =
          row_stats<TPR, NV>(y[0], y[R - 1], mean, mean, k, s_y);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float rho =
            rsqrtf((i ? st.sq_b : st.sq_a) * k.inv_dim + p.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          y[i][j] = fma(y[i][j], rho, -(i ? st.mu_b : st.mu_a) * rho);
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!on[i]) continue;
      if (has_y && group[i] != group_y) {
        group_y = group[i];
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (k.on(j))
            mods.set(j, mul(load8_or(p.gate,
                                     (int64_t)group_y * p.dim + k.at(j), 1.f),
                            load8_or(post ? p.post_weight : nullptr, k.at(j),
                                     1.f)));
      }
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (k.on(j)) {
          x[i][j] = mul(x[i][j], p.residual_scale);
          if (has_y) x[i][j] = fma(y[i][j], mods.get(j), x[i][j]);
          if (p.r != nullptr)
            store8(static_cast<TR*>(p.r),
                   (int64_t)(rb + i * S::kRows + slot) * p.dim + k.at(j),
                   x[i][j]);
        }
    }
    if (!has_h) continue;
    const bool mean = p.pre == kNormLayer;
    const Stats st = row_stats<TPR, NV>(x[0], x[R - 1], mean, mean, k, s_r);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!on[i]) continue;
      if (group[i] != group_h) {
        group_h = group[i];
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (k.on(j)) {
            const int64_t at = (int64_t)group_h * p.dim + k.at(j);
            mods.set(NV + j, mul(add(load8_or(p.scale, at, 0.f), splat(1.f)),
                                 load8_or(p.pre_weight, k.at(j), 1.f)));
            mods.set(2 * NV + j, load8_or(p.shift, at, 0.f));
          }
      }
      const float rho = rsqrtf((i ? st.sq_b : st.sq_a) * k.inv_dim + p.eps);
      const float back = -(i ? st.mu_b : st.mu_a) * rho;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (k.on(j))
          store8(static_cast<TY*>(p.h),
                 (int64_t)(rb + i * S::kRows + slot) * p.dim + k.at(j),
                 fma(fma(x[i][j], rho, back), mods.get(NV + j),
                     mods.get(2 * NV + j)));
    }
  }
}

template <typename TR, typename TY, int TPR, int NV, int R, bool kAhead,
          int kMinCtas>
cudaError_t launch_v(const NormFwdParams& p, int sms, cudaStream_t stream) {
  using S = Shape<TPR>;
  // One wave of CTAs, each with an equal share of the rows; with few rows
  // each takes a pass of its own.
  const int64_t passes = (p.rows + S::kRows - 1) / S::kRows;
  const int64_t grid = std::min<int64_t>((int64_t)sms * kMinCtas, passes);
  auto kernel = norm_fwd_kernel<TR, TY, TPR, NV, R, kAhead, kMinCtas>;
  constexpr int kSmem = 3 * NV * S::kThreads * 32;
  if (kSmem > 32768) {
    const cudaError_t e = cudaFuncSetAttribute(
        kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(S::kThreads), kSmem,
                    stream, p);
}

// Threads, vectors and rows of a pass, CTAs per SM: a row slot as narrow as its
// columns allow up to a warp, then 8 columns to a thread and one row to a pass
// (16320 rows of 1536: 192 threads and 5 CTAs 37.9 us, 4 of them 39.9, 6 with
// spills 46.2, two rows to a pass 44.9, 96 threads of 16 columns 43.0), from
// 2048 on 16 columns, which leaves fewer warps to exchange with (9000 rows of
// 2048: 38.6 us against 46.7).
template <typename TR, typename TY>
cudaError_t launch_t(const NormFwdParams& p, int sms, cudaStream_t stream) {
  if (p.dim <= 64) return launch_v<TR, TY, 8, 1, 2, true, 4>(p, sms, stream);
  if (p.dim <= 128) return launch_v<TR, TY, 16, 1, 2, true, 4>(p, sms, stream);
  if (p.dim <= 256) return launch_v<TR, TY, 32, 1, 2, true, 4>(p, sms, stream);
  if (p.dim <= 512) return launch_v<TR, TY, 64, 1, 1, true, 12>(p, sms, stream);
  if (p.dim <= 1024) return launch_v<TR, TY, 128, 1, 1, true, 7>(p, sms, stream);
  if (p.dim <= 1536) return launch_v<TR, TY, 192, 1, 1, true, 5>(p, sms, stream);
  if (p.dim <= 2048) return launch_v<TR, TY, 128, 2, 1, true, 4>(p, sms, stream);
  if (p.dim <= 4096) return launch_v<TR, TY, 256, 2, 1, true, 2>(p, sms, stream);
  if (p.dim <= 5120) return launch_v<TR, TY, 320, 2, 1, true, 2>(p, sms, stream);
  return launch_v<TR, TY, 512, 2, 1, true, 1>(p, sms, stream);
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
