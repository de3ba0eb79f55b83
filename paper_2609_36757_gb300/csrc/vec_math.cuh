// Small device helpers shared by the elementwise kernels: packed float32 pairs
// (one instruction for two values on sm_103a) and divisions by a number fixed
// at launch.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace fastvr {

// Division of 32-bit numbers below 2^31 by a divisor fixed at launch.
struct FastDiv {
  uint32_t mul, shift;
};
inline FastDiv make_div(uint32_t d) {
  FastDiv f;
  f.shift = 0;
  while ((1ull << f.shift) < d) ++f.shift;
  // mul = ceil(2^(31 + shift) / d) < 2^32; exact for numbers below 2^31
  f.mul = (uint32_t)(((1ull << (31 + f.shift)) + d - 1) / d);
  return f;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t fast_div(uint32_t n, const FastDiv& f) {
  return (uint32_t)(((uint64_t)n * f.mul) >> (31 + f.shift));
}

// Two float32 values in a 64-bit register.
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(x, x); }
__device__ __forceinline__ void split(F2 a, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v));
}
__device__ __forceinline__ F2 add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r.v)
      : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ float sum(F2 a) {
  float lo, hi;
  split(a, lo, hi);
  return lo + hi;
}

// bfloat16 pairs (low half first) to float32 and back.
__device__ __forceinline__ float bf16_lo(uint32_t w) {
  return __uint_as_float(w << 16);
}
__device__ __forceinline__ float bf16_hi(uint32_t w) {
  return __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t bf16_pack(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t bf16_pack(F2 a) {
  float lo, hi;
  split(a, lo, hi);
  return bf16_pack(lo, hi);
}
#endif

}  // namespace fastvr
