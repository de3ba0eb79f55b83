// Pieces of the online softmax that the tile kernels share: exponentials of a
// score tile's rows in registers, their packing to bfloat16 pairs, row maxima.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace fastvr {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

__device__ __forceinline__ uint64_t f2_pack(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// P = 2^(s * scale_log2 - m) for the 32 columns of s[c] (a packed FFMA per
// pair, one MUFU ex2 per element), packed as 16 bf16 pairs; the row sums go
// to four independent packed accumulators.
__device__ __forceinline__ void exp_pack32(const uint32_t (&sc)[32],
                                           uint64_t sl2x2, uint64_t neg2,
                                           uint32_t (&pk)[16],
                                           uint64_t (&acc)[4]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint64_t x2 = f2_fma(f2_pack(__uint_as_float(sc[2 * i]),
                                       __uint_as_float(sc[2 * i + 1])),
                               sl2x2, neg2);
    float x0, x1;
    f2_unpack(x2, x0, x1);
    const float p0 = ex2(x0), p1 = ex2(x1);
    acc[i & 3] = f2_add(acc[i & 3], f2_pack(p0, p1));
    pk[i] = pack_bf16(p0, p1);
  }
}

__device__ __forceinline__ float acc_total(const uint64_t (&acc)[4]) {
  float a0, a1, b0, b1, c0, c1, d0, d1;
  f2_unpack(acc[0], a0, a1);
  f2_unpack(acc[1], b0, b1);
  f2_unpack(acc[2], c0, c1);
  f2_unpack(acc[3], d0, d1);
  return ((a0 + a1) + (b0 + b1)) + ((c0 + c1) + (d0 + d1));
}

// Mask columns >= valid of s[c] (the ragged end of a segment) and fold the
// row max of s[c] into four independent accumulators.
__device__ __forceinline__ void mask_max32(uint32_t (&sc)[32], int c, int valid,
                                           float (&mx)[4]) {
  if (valid < (c + 1) * 32) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (c * 32 + i >= valid) sc[i] = 0xff800000u;  // -inf
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    mx[i & 3] = max3(mx[i & 3], __uint_as_float(sc[2 * i]),
                     __uint_as_float(sc[2 * i + 1]));
}

}  // namespace fastvr
