// Small device helpers shared by the elementwise kernels: packed float32 pairs
// (one instruction for two values on sm_103a), divisions by a number fixed at
// launch and asynchronous copies to shared memory.
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

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// Asynchronous copy of N bytes to shared memory, zeros when !valid.
template <int N>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src,
                                           bool valid) {
  const int n = valid ? N : 0;
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst),
                 "l"(src), "r"(n)
                 : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst),
                 "l"(src), "n"(N), "r"(n)
                 : "memory");
}
// Asks for bytes (place and number multiples of 16) to be brought to L2.
__device__ __forceinline__ void prefetch_l2(const void* from, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from),
               "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void copy_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
#endif

}  // namespace fastvr
