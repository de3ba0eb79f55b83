// Between two blocks: r = a x + gate o post(y), h = pre(r) o (1 + scale) +
// shift, in one pass over memory.
//
// Bound by memory: x and y are read once, r and h written once (8 bytes per
// element in bfloat16).  A thread owns the same columns of all the rows that
// its CTA takes, so the modulation vectors of a group are read and combined
// once (with a warp to a row they were read again for every row, which kept L1
// busier than memory) and kept in shared memory.  What is left is the exchange
// of a row's sums and the instructions around it, so as many CTAs as fit
// without spilling share an SM; where the rows ahead wait in shared memory
// instead of registers, more of them do.  36.1 us (5.6 TB/s) for 16320 rows of
// 1536 in bfloat16 with a layer norm and no post norm.  This and the times
// below are of calls replayed from a graph, a few per cent below a call's own.
#include <algorithm>

#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

// R rows to a pass (of each row slot).
template <typename TR, typename TY, int TPR, int NV, int R, int kDeep,
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
  constexpr int step = R * S::kRows;  // rows of a pass
  const bool has_y = p.y != nullptr, has_h = p.h != nullptr;
  const bool post = has_y && p.post != kNormNone;
  pdl_wait();

  // Rows rb + i kRows + slot of a pass, x then y: kDeep - 1 passes ahead in
  // shared memory (a row to a CTA), or one ahead in registers (kDeep = 0).
  static_assert(kDeep == 0 || S::kRows == 1, "");
  constexpr int kX = sizeof(TR) / 2, kXY = kX + sizeof(TY) / 2;
  Ring<kDeep, R * NV * kXY> ring = {dyn + 6 * NV * S::kThreads};
  Raw8<TR> xr[kDeep ? 1 : R][NV];
  Raw8<TY> yr[kDeep ? 1 : R][NV];
  auto fetch = [&](int rb, int ahead) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if constexpr (kDeep > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          auto index = [&](int thread) {
            const int row = rb + i, col = k.at(j, thread);
            return row < r1 && col < p.dim ? (int64_t)row * p.dim + col : -1;
          };
          ring.template ask<TR>(ahead, (i * NV + j) * kXY, p.x, index);
          if (has_y)
            ring.template ask<TY>(ahead, (i * NV + j) * kXY + kX, p.y, index);
        }
      } else {
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
    }
    if constexpr (kDeep > 0) copy_commit();
  };
  // mods: gate o post_weight (j), (1 + scale) o pre_weight (NV + j) and shift
  // (2 NV + j) of the group last asked for.
  uint32_t group_y = ~0u, group_h = ~0u;

#pragma unroll
  for (int i = 0; i < (kDeep ? kDeep - 1 : 1); ++i) fetch(r0 + i * step, i);
  // every thread makes every pass (barriers and shuffles inside)
  for (int rb = r0; rb < r1; rb += step) {
    // a pass with one exchange only: its part is not written again before
    // every thread has read it
    if (S::kMany && post != has_h) __syncthreads();
    if constexpr (kDeep > 0) {
      fetch(rb + (kDeep - 1) * step, kDeep - 1);
      ring.wait();
    }
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
        const bool here = on[i] && k.on(j);
        if constexpr (kDeep > 0) {
          const int at = (i * NV + j) * kXY;
          x[i][j] = here ? ring.template get<TR>(at) : splat(0.f);
          y[i][j] = here && has_y ? ring.template get<TY>(at + kX) : splat(0.f);
        } else {
          x[i][j] = here ? xr[i][j].widen() : splat(0.f);
          y[i][j] = here && has_y ? yr[i][j].widen() : splat(0.f);
        }
      }
    }
    if constexpr (kDeep > 0)
      ring.next();
    else
      fetch(rb + step, 0);

    if (post) {
      const bool mean = p.post == kNormLayer;
      const Stats st =
          row_stats<TPR, NV>(y[0], y[R - 1], mean, k, s_y);
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
    const Stats st = row_stats<TPR, NV>(x[0], x[R - 1], mean, k, s_r);
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

template <typename TR, typename TY, int TPR, int NV, int R, int kMaxDeep,
          int kMinCtas>
cudaError_t launch_v(const NormFwdParams& p, int sms, cudaStream_t stream) {
  using S = Shape<TPR>;
  // a thread's bytes per vector, and how many passes fit beside one another
  constexpr int kMods = 96, kPass = 8 * R * (int)(sizeof(TR) + sizeof(TY));
  constexpr int kVectors = NV * S::kThreads;
  constexpr int kFit =
      ring_depth(kMinCtas, kVectors, kMods, kPass, kMaxDeep);
  constexpr int kDeep = kMaxDeep == 0 ? 0 : kFit ? kFit : 2;
  constexpr int kSmem = kVectors * (kMods + kDeep * kPass);
  constexpr int kCtas = kFit || !kDeep ? kMinCtas : kSmBytes / (kSmem + 2048);
  // One wave of CTAs, each with an equal share of the rows; with few rows
  // each takes a pass of its own.
  const int64_t passes = (p.rows + S::kRows - 1) / S::kRows;
  const int64_t grid = std::min<int64_t>((int64_t)sms * kCtas, passes);
  auto kernel = norm_fwd_kernel<TR, TY, TPR, NV, R, kDeep, kMinCtas>;
  if (kSmem > 32768) {
    const cudaError_t e = cudaFuncSetAttribute(
        kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(S::kThreads), kSmem,
                    stream, p);
}

// Threads, vectors and rows of a pass, passes ahead in shared memory (0: one in
// registers), CTAs per SM.  Times in bfloat16 with RMS norms before and after,
// but for 64 columns (float32 residual, layer norm after) and 1536 (a layer
// norm alone).  Rows of up to 256 columns lie side by side in a CTA (277236
// rows of 64: 35.3 us with one row to a thread and 6 CTAs, 40.2 with two and 4,
// 49.5 with rows ahead in shared memory).  From there to 512 eight columns to a
// thread and the next row in registers as well (36000 rows of 512: 25.7 us,
// 30.2 through shared memory), above that through shared memory (against
// registers: 36.4 us and 52.6 for 36000 rows of 520, 27.4 and 30.4 for 18000 of
// 1024, 36.1 and 38.6 for 16320 of 1536 by twos), from 2048 on with 16 columns
// to a thread, which leaves fewer warps to exchange with (29.1 and 38.6 for
// 9000 rows of 2048, 30.9 and 40.9 for 3600 of 5120, 46.3 and 66.5 for 3000 of
// 8192).  A modulation of its own for every row makes the ends of groups count:
// one row at a time and in registers then (8160 rows of 1536: 43.0 us and
// 45.3).
template <typename TR, typename TY>
cudaError_t launch_t(const NormFwdParams& p, int sms, cudaStream_t stream) {
  if (p.dim <= 64) return launch_v<TR, TY, 8, 1, 1, 0, 6>(p, sms, stream);
  if (p.dim <= 128) return launch_v<TR, TY, 16, 1, 1, 0, 6>(p, sms, stream);
  if (p.dim <= 256) return launch_v<TR, TY, 32, 1, 1, 0, 6>(p, sms, stream);
  if (p.dim <= 512) return launch_v<TR, TY, 64, 1, 1, 0, 16>(p, sms, stream);
  if (p.dim <= 768) return launch_v<TR, TY, 96, 1, 1, 2, 9>(p, sms, stream);
  if (p.dim <= 1024) return launch_v<TR, TY, 128, 1, 1, 2, 8>(p, sms, stream);
  if (p.dim <= 1536 && p.group_tokens < kFewTokens)
    return launch_v<TR, TY, 192, 1, 1, 0, 5>(p, sms, stream);
  if (p.dim <= 1536) return launch_v<TR, TY, 192, 1, 2, 2, 4>(p, sms, stream);
  if (p.dim <= 2048) return launch_v<TR, TY, 128, 2, 1, 4, 5>(p, sms, stream);
  if (p.dim <= 4096) return launch_v<TR, TY, 256, 2, 1, 3, 2>(p, sms, stream);
  if (p.dim <= 5120) return launch_v<TR, TY, 320, 2, 1, 3, 2>(p, sms, stream);
  return launch_v<TR, TY, 512, 2, 1, 3, 1>(p, sms, stream);
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
