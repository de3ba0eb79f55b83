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

// Sums of N values over the TPR threads of a row, the same on each of them;
// the order of the additions is fixed.  smem: N * TPR / 32 floats, used when
// a row has more than a warp (the CTA then has exactly one row).
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* smem) {
#pragma unroll
  for (int m = 16; m > 0; m >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], m);
  if constexpr (TPR > 32) {
    constexpr int kWarps = TPR / 32;
    const int warp = threadIdx.x / 32;
    __syncthreads();  // the previous sums have been read
    if (threadIdx.x % 32 == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) smem[i * kWarps + warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v[i] += smem[i * kWarps + w];
    }
  }
}

}  // namespace norm
}  // namespace fastvr
