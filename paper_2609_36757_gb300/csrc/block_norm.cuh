// Shared by the forward and the backward of the gated residual and norms.
#pragma once

#include <cuda_bf16.h>

#include "fastvr_internal.h"

namespace fastvr {
namespace norm {

// 8 consecutive elements in memory: 16 bytes of bfloat16 or 32 of float32.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const void* base, int64_t i) {
    u = *reinterpret_cast<const uint4*>(
        static_cast<const __nv_bfloat16*>(base) + i);
  }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(w[e] << 16);
      f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* base, int64_t i) {
    const float4* p =
        reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
    a = p[0];
    b = p[1];
  }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
    f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  }
};

__device__ __forceinline__ void store8(__nv_bfloat16* base, int64_t i,
                                       const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&v);
  }
  *reinterpret_cast<uint4*>(base + i) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* base, int64_t i,
                                       const float (&f)[8]) {
  float4* p = reinterpret_cast<float4*>(base + i);
  p[0] = make_float4(f[0], f[1], f[2], f[3]);
  p[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// 8 floats of an optional vector, `absent` where there is none.
__device__ __forceinline__ void load8_or(const float* base, int64_t i,
                                         float absent, float (&f)[8]) {
  if (base == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = absent;
    return;
  }
  Raw8<float> r;
  r.load(base, i);
  r.widen(f);
}

__device__ __forceinline__ float sum8(const float (&f)[8]) {
  return ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
}

// Sums of a and of b over the L lanes of a row within a warp, at the price of
// about one: the halves of the lanes first trade what they do not keep.
// `keep_sums` leaves a's sum on the lanes of the lower half and b's on those
// of the upper one; `both_sums` leaves both on every lane.
template <int L>
__device__ __forceinline__ float keep_sums(float a, float b) {
  const bool hi = threadIdx.x & (L / 2);
  float v = hi ? b : a;
  v += __shfl_xor_sync(0xffffffffu, hi ? a : b, L / 2);
#pragma unroll
  for (int m = L / 4; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
template <int L>
__device__ __forceinline__ void both_sums(float& a, float& b) {
  const bool hi = threadIdx.x & (L / 2);
  const float v = keep_sums<L>(a, b);
  const float o = __shfl_xor_sync(0xffffffffu, v, L / 2);
  a = hi ? o : v;
  b = hi ? v : o;
}

// A row's threads, 8 columns each: TPR of them.  Up to 32: 128 / TPR rows side
// by side in a CTA of 128 threads, their sums within a warp.  Above: one row
// to a CTA of (at most) TPR threads, its sums across the warps.
template <int TPR>
struct Shape {
  static constexpr int kThreads = TPR <= 32 ? 128 : TPR;
  static constexpr int kLanes = TPR < 32 ? TPR : 32;
  static constexpr int kRows = TPR <= 32 ? 128 / TPR : 1;
  static constexpr bool kMany = TPR > 32;
  static constexpr int kWarps = kMany ? TPR / 32 : 1;
};

// What a thread knows of its row's columns.
struct Cols {
  int c;           // first of its 8 columns
  bool on;         // they exist
  int warps;       // warps of the row
  float inv_dim, inv_warp;  // 1 / columns of the row, of this warp
  float last;      // columns of the row's last warp
};
template <int TPR>
__device__ __forceinline__ Cols make_cols(int dim) {
  using S = Shape<TPR>;
  Cols k;
  k.c = (S::kRows > 1 ? threadIdx.x % TPR : threadIdx.x) * 8;
  k.on = k.c < dim;
  k.warps = S::kMany ? blockDim.x / 32 : 1;
  k.inv_dim = 1.f / (float)dim;
  const int warp = S::kMany ? threadIdx.x / 32 : 0;
  k.inv_warp = 1.f / (float)min(S::kMany ? 256 : dim, dim - warp * 256);
  k.last = (float)(dim - (k.warps - 1) * 256);
  return k;
}

// Sums over the row of a and of b, on every thread; `part` (kWarps entries)
// is this exchange's own: two exchanges with another part between them need
// one barrier each.
template <int TPR>
__device__ __forceinline__ void row_sums(float& a, float& b, const Cols& k,
                                         float2* part) {
  using S = Shape<TPR>;
  if constexpr (!S::kMany) {
    both_sums<S::kLanes>(a, b);
  } else {
    const float v = keep_sums<32>(a, b);
    if (threadIdx.x % 16 == 0)
      reinterpret_cast<float*>(part)[threadIdx.x / 16] = v;
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < S::kWarps; ++w)
      if (w < k.warps) {
        const float2 x = part[w];
        a += x.x;
        b += x.y;
      }
  }
}

// Mean (0 where it is not wanted) and sum of squared deviations of two rows,
// 8 columns per thread (zeros where !k.on), on every thread.  Two passes over
// the warp's registers; the warps' parts are then put together: their own
// squares, and what their means differ from the row's.
struct Stats {
  float mu_a, mu_b, sq_a, sq_b;
};
template <int TPR>
__device__ __forceinline__ Stats row_stats(const float (&a)[8],
                                           const float (&b)[8], bool mean_a,
                                           bool mean_b, const Cols& k,
                                           float4* part) {
  using S = Shape<TPR>;
  Stats st;
  st.mu_a = st.mu_b = 0.f;
  if (mean_a || mean_b) {
    st.mu_a = mean_a ? sum8(a) : 0.f;
    st.mu_b = mean_b ? sum8(b) : 0.f;
    both_sums<S::kLanes>(st.mu_a, st.mu_b);
    st.mu_a *= k.inv_warp;
    st.mu_b *= k.inv_warp;
  }
  st.sq_a = st.sq_b = 0.f;
  if (k.on) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = a[e] - st.mu_a, y = b[e] - st.mu_b;
      st.sq_a = fmaf(x, x, st.sq_a);
      st.sq_b = fmaf(y, y, st.sq_b);
    }
  }
  if constexpr (!S::kMany) {
    both_sums<S::kLanes>(st.sq_a, st.sq_b);
  } else {
    const float v = keep_sums<32>(st.sq_a, st.sq_b);
    if (threadIdx.x % 16 == 0)  // lane 0: of a, lane 16: of b
      reinterpret_cast<float2*>(part)[threadIdx.x / 16] =
          make_float2(threadIdx.x & 16 ? st.mu_b : st.mu_a, v);
    __syncthreads();
    float sa = 0.f, sb = 0.f;
    st.sq_a = st.sq_b = 0.f;
#pragma unroll
    for (int w = 0; w < S::kWarps; ++w)
      if (w < k.warps) {
        const float4 x = part[w];
        const float n = w == k.warps - 1 ? k.last : 256.f;
        sa = fmaf(n, x.x, sa);
        sb = fmaf(n, x.z, sb);
        st.sq_a += x.y;
        st.sq_b += x.w;
      }
    if (mean_a || mean_b) {
      st.mu_a = sa * k.inv_dim;
      st.mu_b = sb * k.inv_dim;
#pragma unroll
      for (int w = 0; w < S::kWarps; ++w)
        if (w < k.warps) {
          const float n = w == k.warps - 1 ? k.last : 256.f;
          const float4 x = part[w];
          const float da = x.x - st.mu_a, db = x.z - st.mu_b;
          st.sq_a = fmaf(n * da, da, st.sq_a);
          st.sq_b = fmaf(n * db, db, st.sq_b);
        }
    }
  }
  return st;
}

// Threads of a row for dim columns (8 each): 8, 16, or whole warps.
inline int row_threads(int dim) {
  const int n = dim / 8;
  return n <= 8 ? 8 : n <= 16 ? 16 : (n + 31) / 32 * 32;
}

}  // namespace norm
}  // namespace fastvr
